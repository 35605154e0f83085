// Backward pass of attention over packed sequences (packed.hpp has the formulas), in two passes that take the
// weights again from the scores and the forward pass's log-sum-exp:
//   dq      queries resident, keys and values streamed; also leaves delta for the other pass
//   dk, dv  keys resident, the queries of every head that shares them streamed, one head after another: their sums
//           need no atomics, and come out in one order
#include "packed.hpp"

namespace gformer {
namespace {

template <typename T, int D> __global__ __launch_bounds__(kPackedThreads) void packed_dq_kernel(PackedArgs a, int tiles) {
  using P = Products<T, D>;
  constexpr int R = P::R, ROW = P::ROW, NS = R / 32, MT = D / 32;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  auto& sm = *reinterpret_cast<PackedTiles<T, D>*>(smem_raw);
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
  for (int t = 0; t < n_tiles; ++t) {
    const int t0 = t * R;
    T *kt = sm.x[t & 1], *vt = sm.y[t & 1];
    const bool cut = t0 + R - 1 > i0 + off;
    ks.template store<ROW>(kt, tid);
    vs.template store<ROW>(vt, tid);
    if (cut && ks.odd()) sm.odd[t % 3] = 1;
    if (tid == 0) sm.odd[(t + 1) % 3] = 0;
    lds_barrier();
    if (t + 1 < n_tiles) {
      ks.load(kp, a.ks[0], t0 + R, nk - 1, tid);
      vs.load(vp, a.vs[0], t0 + R, nk - 1, tid);
    }
    if (t0 > min(q0 + 31, nq - 1) + off) continue;
    const bool mask = t0 + R - 1 > q0 + off, by_rows = mask && sm.odd[t % 3];
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      const f32x16 s = P::scores(kt + 32 * n * ROW, q, lane), dp = P::scores(vt + 32 * n * ROW, g, lane);
      float ds[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        ds[r] = __builtin_amdgcn_exp2f(fmaf(s[r], sc, -lse)) * (dp[r] - delta);
        if (mask && t0 + 32 * n + 8 * (r / 4) + 4 * lh + r % 4 > seen) ds[r] = 0.f;
      }
      const typename P::Weights w = P::weights(ds);
      if (by_rows) P::product_by_rows(dq, kt + 32 * n * ROW, w, 0, seen + 1 - t0 - 32 * n, lane);
      else P::product(dq, kt + 32 * n * ROW, w, lane);
    }
  }
  lds_barrier();
  if (q0 < nq)
    put_rows<T, D>(dq, a.scale, reinterpret_cast<T*>(smem_raw) + wave * 32 * ROW, rows_of<T>(a.dq, a.dqs, qbase + q0, h), a.dqs[0],
                   min(32, nq - q0), lane);
}

template <typename T, int D> __global__ __launch_bounds__(kPackedThreads, 1) void packed_dkdv_kernel(PackedArgs a, int tiles) {
  using P = Products<T, D>;
  constexpr int R = P::R, ROW = P::ROW, NS = R / 32, MT = D / 32;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  auto& sm = *reinterpret_cast<PackedTiles<T, D>*>(smem_raw);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, ln = lane & 31, lh = lane >> 5;

  // first tiles first: the most queries see them
  const int kvh = blockIdx.x % a.Hkv;
  const SeqTile at = find_tile<kPackedRows>(a.cu_k, a.n_seqs, a.total_k, blockIdx.x / a.Hkv, lane);
  if (at.first < 0) return;
  const int kbase = packed_row(a.cu_k, at.seq, a.total_k), j0 = at.first;
  if (at.seq == a.n_seqs) {
    if (a.zero_tail && j0 < a.total_k - kbase) {
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
  if (total) load(0);
  if (tid < 3) sm.odd[tid] = 0;
  lds_barrier();
  for (int it = 0; it < total; ++it) {
    const int t0 = (first_tile + it % per_head) * R;
    T *qt = sm.x[it & 1], *gt = sm.y[it & 1];
    const bool end = t0 + R > nq;
    const bool cut = end || t0 < min(j0 + kPackedRows, nk) - 1 - off;
    qs.template store<ROW>(qt, tid);
    gs.template store<ROW>(gt, tid);
    if (tid < R) sm.lse[it & 1][tid] = stat;
    else if (tid < 2 * R) sm.delta[it & 1][tid - R] = stat;
    if (cut && (qs.odd() || gs.odd())) sm.odd[it % 3] = 1;
    if (tid == 0) sm.odd[(it + 1) % 3] = 0;
    lds_barrier();
    if (it + 1 < total) load(it + 1);
    if (k0 >= nk || t0 + R - 1 < k0 - off) continue;   // no key here, or none that a query of the tile sees
    const bool mask = end || t0 < min(k0 + 31, nk - 1) - off, by_rows = mask && sm.odd[it % 3];
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      const f32x16 s = P::scores(qt + 32 * n * ROW, k, lane), dp = P::scores(gt + 32 * n * ROW, v, lane);
      const float* lse = sm.lse[it & 1] + 32 * n + 4 * lh;
      const float* delta = sm.delta[it & 1] + 32 * n + 4 * lh;
      float p[16], ds[16];
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4_t l4 = *reinterpret_cast<const f32x4_t*>(lse + 8 * g), d4 = *reinterpret_cast<const f32x4_t*>(delta + 8 * g);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * g + e;
          p[r] = __builtin_amdgcn_exp2f(fmaf(s[r], sc, -l4[e]));
          ds[r] = p[r] * (dp[r] - d4[e]);
          const int i = t0 + 32 * n + 8 * g + 4 * lh + e;
          if (mask && (i < from || i >= nq)) p[r] = ds[r] = 0.f;
        }
      }
      const typename P::Weights wp = P::weights(p), wd = P::weights(ds);
      const int lo = from - t0 - 32 * n, hi = nq - t0 - 32 * n;
      if (by_rows) {
        P::product_by_rows(dv, gt + 32 * n * ROW, wp, lo, hi, lane);
        P::product_by_rows(dk, qt + 32 * n * ROW, wd, lo, hi, lane);
      } else {
        P::product(dv, gt + 32 * n * ROW, wp, lane);
        P::product(dk, qt + 32 * n * ROW, wd, lane);
      }
    }
  }
  lds_barrier();
  if (k0 < nk) {
    T* own = reinterpret_cast<T*>(smem_raw) + wave * 32 * ROW;
    put_rows<T, D>(dk, a.scale, own, rows_of<T>(a.dk, a.dks, kbase + k0, kvh), a.dks[0], min(32, nk - k0), lane);
    put_rows<T, D>(dv, 1.f, own, rows_of<T>(a.dv, a.dvs, kbase + k0, kvh), a.dvs[0], min(32, nk - k0), lane);
  }
}

template <typename T, int D> hipError_t launch(const PackedArgs& a, hipStream_t s) {
  const size_t smem = sizeof(PackedTiles<T, D>);
  auto dq = packed_dq_kernel<T, D>;
  auto dkdv = packed_dkdv_kernel<T, D>;
  if (hipError_t e = allow_lds(dq, smem); e != hipSuccess) return e;
  if (hipError_t e = allow_lds(dkdv, smem); e != hipSuccess) return e;
  const int64_t qt = packed_tiles(a.total_q, a.n_seqs, kPackedRows), kt = packed_tiles(a.total_k, a.n_seqs, kPackedRows);
  dq<<<dim3((unsigned)(qt * a.H)), dim3(kPackedThreads), smem, s>>>(a, (int)qt);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  dkdv<<<dim3((unsigned)(kt * a.Hkv)), dim3(kPackedThreads), smem, s>>>(a, (int)kt);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_bwd(const PackedArgs& a, bool bf16, hipStream_t s) {
  if (bf16) return a.d == 128 ? launch<uint16_t, 128>(a, s) : launch<uint16_t, 64>(a, s);
  return a.d == 128 ? launch<float, 128>(a, s) : launch<float, 64>(a, s);
}

}  // namespace gformer
