// Backward pass of attention over packed sequences (packed.hpp has the formulas), in two passes that take the
// weights again from the scores and the forward pass's log-sum-exp:
//   dq      queries resident, keys and values streamed; also leaves delta for the other pass
//   dk, dv  keys resident, the queries of every head that shares them streamed, one head after another: their sums
//           need no atomics, and come out in one order
#include "packed.hpp"

namespace gformer {
namespace {

// waves on a SIMD that the kernels' registers are kept down for
template <typename T, int D> constexpr int kWaves = sizeof(T) == 4 && D == 128 ? 1 : 2;
// keys per tile of the dq pass
template <typename T, int D> constexpr int kKeyTile = sizeof(T) == 2 && D == 64 ? 64 : 32;
constexpr int kQueryTile = 32;   // queries per tile of the dk, dv pass
// That pass's workgroups take the query tiles of their keys in this many streams, four waves each, whose sums are joined at
// the end.  A causal sequence's first keys are seen by all its queries, its last by few, and there are only as many workgroups as
// key tiles and key heads: the longest one decides, and with two streams it takes half as long.
template <typename T, int D> constexpr int kStreams = kWaves<T, D>;
// its value rows stay in LDS where their registers are wanted for the sums
template <typename T, int D> constexpr bool kValuesInLds = sizeof(T) == 2 && D == 128;
template <typename T, int D> using DqTiles = PackedTiles<T, kKeyTile<T, D>, Products<T, D>::BOTH, Products<T, D>::BY_ROWS>;
template <typename T, int D> struct KeyTiles {
  PackedTiles<T, kQueryTile, Products<T, D>::BOTH, Products<T, D>::BOTH> stream[kStreams<T, D>];
  T v[kValuesInLds<T, D> ? kPackedRows * Products<T, D>::BY_ROWS : 1];
};

template <typename T, int D> __global__ __launch_bounds__(kPackedThreads, (kWaves<T, D>)) void packed_dq_kernel(PackedArgs a, int tiles) {
  using P = Products<T, D>;
  constexpr int R = kKeyTile<T, D>, KROW = P::BOTH, VROW = P::BY_ROWS, NS = R / 32, MT = D / 32;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  auto& sm = *reinterpret_cast<DqTiles<T, D>*>(smem_raw);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, ln = lane & 31, lh = lane >> 5;

  const int hh = blockIdx.x % a.H, kvh = hh % a.Hkv, h = kvh * (a.H / a.Hkv) + hh / a.Hkv;
  const SeqTile at = find_tile<kPackedRows>(a.cu_q, a.n_seqs, a.total_q, tiles - 1 - blockIdx.x / a.H, lane);
  if (at.first < 0) return;
  const int qbase = packed_row(a.cu_q, at.seq, a.total_q), i0 = at.first;
  if (at.seq == a.n_seqs) {
    if (a.zero_tail && i0 < a.total_q - qbase)
      zero_rows<T, D>(rows_of<T>(a.dq, a.dqs, qbase + i0, h), a.dqs[0], min(kPackedRows, a.total_q - qbase - i0), tid);
    return;
  }
  const int nq = packed_row(a.cu_q, at.seq + 1, a.total_q) - qbase;
  if (i0 >= nq) return;
  const int kbase = packed_row(a.cu_k, at.seq, a.total_k);
  const int nk = max(packed_row(a.cu_k, at.seq + 1, a.total_k) - kbase, 0), off = nk - nq;

  const int q0 = i0 + 32 * wave, i = q0 + ln, ic = min(i, nq - 1), seen = ic + off;
  typename P::Resident q, g;
  P::load(g, rows_of<T>((const void*)a.out, a.os, qbase + ic, h), lane, false);
  P::load(q, rows_of<T>(a.dout, a.gs, qbase + ic, h), lane, false);
  const float delta = P::dot(q, g);
  g = q;
  P::load(q, rows_of<T>(a.q, a.qs, qbase + ic, h), lane, a.scale < 0.f);
  const int64_t stat = (int64_t)h * a.total_q + qbase + ic;
  if (lh == 0 && i < nq) a.delta[stat] = delta;
  const float lse = a.lse[stat] * kLog2e;
  const float sc = (a.scale == 0.f ? 1e-30f : fabsf(a.scale)) * kLog2e;

  f32x16 dq[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int r = 0; r < 16; ++r) dq[mt][r] = 0.f;

  const T* kp = rows_of<T>(a.k, a.ks, kbase, kvh);
  const T* vp = rows_of<T>(a.v, a.vs, kbase, kvh);
  const int last_key = min(i0 + kPackedRows, nq) - 1 + off;
  const int n_tiles = last_key < 0 ? 0 : last_key / R + 1;
  Stage<T, D, R> ks, vs;
  if (n_tiles) {
    ks.load(kp, a.ks[0], 0, nk - 1, tid);
    vs.load(vp, a.vs[0], 0, nk - 1, tid);
  }
  if (tid < 3) sm.odd[tid] = 0;
  lds_barrier();
  auto sums = [&](int t, auto mask_tag) {
    constexpr bool MASK = decltype(mask_tag)::value;
    const int t0 = t * R;
    const T *kt = sm.x[t & 1], *vt = sm.y[t & 1];
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      const f32x16 s = P::template scores<KROW>(kt + 32 * n * KROW, q, lane), dp = P::template scores<VROW>(vt + 32 * n * VROW, g, lane);
      float ds[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        ds[r] = __builtin_amdgcn_exp2f(fmaf(s[r], sc, -lse)) * (dp[r] - delta);
        if (MASK && t0 + 32 * n + 8 * (r / 4) + 4 * lh + r % 4 > seen) ds[r] = 0.f;
      }
      const typename P::Weights w = P::weights(ds);
      if (MASK && sm.odd[t % 3]) P::template product_by_rows<KROW>(dq, kt + 32 * n * KROW, w, 0, seen + 1 - t0 - 32 * n, lane);
      else P::template product<KROW>(dq, kt + 32 * n * KROW, w, lane);
    }
  };
  for (int t = 0; t < n_tiles; ++t) {
    const int t0 = t * R;
    ks.template store<KROW>(sm.x[t & 1], tid);
    vs.template store<VROW>(sm.y[t & 1], tid);
    if (t0 + R - 1 > i0 + off && ks.odd()) sm.odd[t % 3] = 1;   // some query of the workgroup does not see the whole tile
    if (tid == 0) sm.odd[(t + 1) % 3] = 0;
    lds_barrier();
    if (t + 1 < n_tiles) {
      ks.load(kp, a.ks[0], t0 + R, nk - 1, tid);
      vs.load(vp, a.vs[0], t0 + R, nk - 1, tid);
    }
    if (t0 > min(q0 + 31, nq - 1) + off) continue;
    if (t0 + R - 1 > q0 + off) sums(t, std::true_type{});
    else sums(t, std::false_type{});
  }
  lds_barrier();
  if (q0 < nq)
    put_rows<T, D>(dq, a.scale, reinterpret_cast<T*>(smem_raw) + wave * 32 * VROW, rows_of<T>(a.dq, a.dqs, qbase + q0, h), a.dqs[0],
                   min(32, nq - q0), lane);
}

template <typename T, int D> __global__ __launch_bounds__((kPackedThreads * kStreams<T, D>), (kWaves<T, D>)) void packed_dkdv_kernel(PackedArgs a, int tiles) {
  using P = Products<T, D>;
  constexpr int R = kQueryTile, ROW = P::BOTH, NS = R / 32, MT = D / 32;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  constexpr int S = kStreams<T, D>;
  auto& all = *reinterpret_cast<KeyTiles<T, D>*>(smem_raw);
  const int stream = __builtin_amdgcn_readfirstlane(threadIdx.x / kPackedThreads);
  auto& sm = all.stream[stream];
  const int tid = threadIdx.x % kPackedThreads, lane = tid & 63, wave = tid >> 6, ln = lane & 31, lh = lane >> 5;

  // first tiles first: the most queries see them
  const int kvh = blockIdx.x % a.Hkv;
  const SeqTile at = find_tile<kPackedRows>(a.cu_k, a.n_seqs, a.total_k, blockIdx.x / a.Hkv, lane);
  if (at.first < 0) return;
  const int kbase = packed_row(a.cu_k, at.seq, a.total_k), j0 = at.first;
  if (at.seq == a.n_seqs) {
    if (a.zero_tail && stream == 0 && j0 < a.total_k - kbase) {
      const int rows = min(kPackedRows, a.total_k - kbase - j0);
      zero_rows<T, D>(rows_of<T>(a.dk, a.dks, kbase + j0, kvh), a.dks[0], rows, tid);
      zero_rows<T, D>(rows_of<T>(a.dv, a.dvs, kbase + j0, kvh), a.dvs[0], rows, tid);
    }
    return;
  }
  const int nk = packed_row(a.cu_k, at.seq + 1, a.total_k) - kbase;
  if (j0 >= nk) return;
  const int qbase = packed_row(a.cu_q, at.seq, a.total_q);
  const int nq = max(packed_row(a.cu_q, at.seq + 1, a.total_q) - qbase, 0), off = nk - nq;

  const int k0 = j0 + 32 * wave, j = k0 + ln, jc = min(j, nk - 1);
  const int from = jc - off;   // the first query that sees this lane's key
  typename P::Resident k, v;
  P::load(k, rows_of<T>(a.k, a.ks, kbase + jc, kvh), lane, a.scale < 0.f);
  P::load(v, rows_of<T>(a.v, a.vs, kbase + jc, kvh), lane, false);
  T* const own_v = all.v + (kValuesInLds<T, D> ? wave * 32 * P::BY_ROWS : 0);
  if constexpr (kValuesInLds<T, D>)
    if (stream == 0) P::to_lds(v, own_v, lane);   // read behind the first barrier
  const float sc = (a.scale == 0.f ? 1e-30f : fabsf(a.scale)) * kLog2e;

  f32x16 dk[MT], dv[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int r = 0; r < 16; ++r) dk[mt][r] = dv[mt][r] = 0.f;

  // the tiles of queries that see any of the workgroup's keys, for every head of the group in turn
  const int first_tile = max(j0 - off, 0) / R;
  const int per_head = nq == 0 ? 0 : (nq - 1) / R + 1 - first_tile, G = a.H / a.Hkv, total = max(per_head, 0) * G;
  Stage<T, D, R> qs, gs;
  float stat = 0.f;   // threads 0 .. R-1: lse of a query, R .. 2R-1: delta
  auto load = [&](int it) {
    const int h = kvh * G + it / per_head, t0 = (first_tile + it % per_head) * R;
    qs.load(rows_of<T>(a.q, a.qs, qbase, h), a.qs[0], t0, nq - 1, tid);
    gs.load(rows_of<T>(a.dout, a.gs, qbase, h), a.gs[0], t0, nq - 1, tid);
    const int64_t at_stat = (int64_t)h * a.total_q + qbase;
    if (tid < R) stat = a.lse[at_stat + min(t0 + tid, nq - 1)] * kLog2e;
    else if (tid < 2 * R) stat = a.delta[at_stat + min(t0 + tid - R, nq - 1)];
  };
  if (stream < total) load(stream);
  if (tid < 3) sm.odd[tid] = 0;
  lds_barrier();
  auto sums = [&](int it, int t0, auto mask_tag) {   // tile number `it` of the stream
    constexpr bool MASK = decltype(mask_tag)::value;
    const T *qt = sm.x[it & 1], *gt = sm.y[it & 1];
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      const float* lse = sm.lse[it & 1] + 32 * n + 4 * lh;
      const float* delta = sm.delta[it & 1] + 32 * n + 4 * lh;
      const int lo = from - t0 - 32 * n, hi = nq - t0 - 32 * n;   // rows that see this lane's key
      float p[16], ds[16];
      const f32x16 s = P::template scores<ROW>(qt + 32 * n * ROW, k, lane);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4_t l4 = *reinterpret_cast<const f32x4_t*>(lse + 8 * g);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = 8 * g + 4 * lh + e;
          p[4 * g + e] = __builtin_amdgcn_exp2f(fmaf(s[4 * g + e], sc, -l4[e]));
          if (MASK && (i < lo || i >= hi)) p[4 * g + e] = 0.f;
        }
      }
      f32x16 dp;
      if constexpr (kValuesInLds<T, D>) dp = P::template scores_lds<ROW>(gt + 32 * n * ROW, own_v, lane);
      else dp = P::template scores<ROW>(gt + 32 * n * ROW, v, lane);
      const typename P::Weights wp = P::weights(p);
      if (MASK && sm.odd[it % 3]) P::template product_by_rows<ROW>(dv, gt + 32 * n * ROW, wp, lo, hi, lane);
      else P::template product<ROW>(dv, gt + 32 * n * ROW, wp, lane);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4_t d4 = *reinterpret_cast<const f32x4_t*>(delta + 8 * g);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = 8 * g + 4 * lh + e;
          ds[4 * g + e] = p[4 * g + e] * (dp[4 * g + e] - d4[e]);
          if (MASK && (i < lo || i >= hi)) ds[4 * g + e] = 0.f;
        }
      }
      const typename P::Weights wd = P::weights(ds);
      if (MASK && sm.odd[it % 3]) P::template product_by_rows<ROW>(dk, qt + 32 * n * ROW, wd, lo, hi, lane);
      else P::template product<ROW>(dk, qt + 32 * n * ROW, wd, lane);
    }
  };
  for (int it = stream, n = 0; it - stream < total; it += S, ++n) {   // the streams meet at every barrier
    const bool on = it < total;
    const int t0 = on ? (first_tile + it % per_head) * R : 0;
    const bool end = t0 + R > nq;
    if (on) {
      qs.template store<ROW>(sm.x[n & 1], tid);
      gs.template store<ROW>(sm.y[n & 1], tid);
      if (tid < R) sm.lse[n & 1][tid] = stat;
      else if (tid < 2 * R) sm.delta[n & 1][tid - R] = stat;
      if ((end || t0 < min(j0 + kPackedRows, nk) - 1 - off) && (qs.odd() || gs.odd())) sm.odd[n % 3] = 1;
    }
    if (tid == 0) sm.odd[(n + 1) % 3] = 0;
    lds_barrier();
    if (it + S < total) load(it + S);
    if (!on || k0 >= nk || t0 + R - 1 < k0 - off) continue;   // no key here, or none that a query of the tile sees
    if (end || t0 < min(k0 + 31, nk - 1) - off) sums(n, t0, std::true_type{});
    else sums(n, t0, std::false_type{});
  }
  lds_barrier();
  if constexpr (S > 1) {
    // the second stream's sums, a register of 64 lanes at a time
    static_assert(S == 2 && sizeof(KeyTiles<T, D>) >= kPackedRows * D * sizeof(float));
    float* own = reinterpret_cast<float*>(smem_raw) + wave * 32 * D + lane;
    auto join = [&](f32x16 (&sum)[MT]) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (stream) own[64 * (16 * mt + r)] = sum[mt][r];
      lds_barrier();
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (!stream) sum[mt][r] += own[64 * (16 * mt + r)];
      lds_barrier();
    };
    join(dk);
    join(dv);
    if (stream) return;
  }
  if (k0 < nk) {
    T* own = reinterpret_cast<T*>(smem_raw) + wave * 32 * P::BY_ROWS;
    put_rows<T, D>(dk, a.scale, own, rows_of<T>(a.dk, a.dks, kbase + k0, kvh), a.dks[0], min(32, nk - k0), lane);
    put_rows<T, D>(dv, 1.f, own, rows_of<T>(a.dv, a.dvs, kbase + k0, kvh), a.dvs[0], min(32, nk - k0), lane);
  }
}

template <typename T, int D> hipError_t launch(const PackedArgs& a, hipStream_t s) {
  const size_t dq_smem = sizeof(DqTiles<T, D>), dkdv_smem = sizeof(KeyTiles<T, D>);
  auto dq = packed_dq_kernel<T, D>;
  auto dkdv = packed_dkdv_kernel<T, D>;
  if (hipError_t e = allow_lds(dq, dq_smem); e != hipSuccess) return e;
  if (hipError_t e = allow_lds(dkdv, dkdv_smem); e != hipSuccess) return e;
  const int64_t qt = packed_tiles(a.total_q, a.n_seqs, kPackedRows), kt = packed_tiles(a.total_k, a.n_seqs, kPackedRows);
  dq<<<dim3((unsigned)(qt * a.H)), dim3(kPackedThreads), dq_smem, s>>>(a, (int)qt);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  dkdv<<<dim3((unsigned)(kt * a.Hkv)), dim3(kPackedThreads * kStreams<T, D>), dkdv_smem, s>>>(a, (int)kt);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_bwd(const PackedArgs& a, bool bf16, hipStream_t s) {
  if (bf16) return a.d == 128 ? launch<uint16_t, 128>(a, s) : launch<uint16_t, 64>(a, s);
  return a.d == 128 ? launch<float, 128>(a, s) : launch<float, 64>(a, s);
}

}  // namespace gformer
