// Backward pass of attention over packed sequences (packed.hpp has the formulas), in two passes that take the
// weights again from the scores and the forward pass's log-sum-exp:
//   dq      queries resident, keys and values streamed; also leaves both statistics of a query for the other pass
//   dk, dv  keys resident, the queries of every head that shares them streamed, one head after another: their sums
//           need no atomics, and come out in one order
#include "packed.hpp"

namespace gformer {
namespace {

// waves on a SIMD that the kernels' registers are kept down for
template <typename T, int D> constexpr int kWaves = sizeof(T) == 4 && D == 128 ? 1 : 2;
// keys per tile of the dq pass
template <typename T, int D> constexpr int kKeyTile = sizeof(T) == 2 && D == 64 ? 64 : 32;
// queries per tile of the dk, dv pass
template <typename T, int D> constexpr int kQueryTile = sizeof(T) == 2 && D == 64 ? 64 : 32;
// That pass's workgroups take the query tiles of their keys in this many streams, four waves each, whose sums are joined at
// the end.  A causal sequence's first keys are seen by all its queries, its last by few, and there are only as many workgroups as
// key tiles and key heads: the longest one decides, and with two streams it takes half as long.
template <typename T, int D> constexpr int kStreams = kWaves<T, D>;
// its value rows stay in LDS where their registers are wanted for the sums
template <typename T, int D> constexpr bool kValuesInLds = sizeof(T) == 2 && D == 128;
constexpr int kBuffers = 3;      // tiles in LDS: one in use, two on their way
template <typename T, int D> struct alignas(256) DqTiles {
  T k[kBuffers][kKeyTile<T, D> * D], v[kBuffers][kKeyTile<T, D> * D];
  int flag;
};
template <typename T, int D> struct alignas(256) QueryTiles {
  T q[kBuffers][kQueryTile<T, D> * D], g[kBuffers][kQueryTile<T, D> * D];
  float stats[kBuffers][2 * kQueryTile<T, D>];   // in base 2: lse of the queries, then -delta
};
template <typename T, int D> struct alignas(256) KeyTiles {
  QueryTiles<T, D> stream[kStreams<T, D>];
  T v[kValuesInLds<T, D> ? kPackedRows * D : 8];
  int flag;
};

template <typename T, int D> __global__ __launch_bounds__(kPackedThreads, (kWaves<T, D>)) void packed_dq_kernel(PackedArgs a, int tiles) {
  using P = Products<T, D>;
  constexpr int R = kKeyTile<T, D>, NS = R / 32, MT = D / 32, W = kPackedThreads / 64;
  using L = Tile<T, D, R>;
  extern __shared__ __align__(256) unsigned char smem_raw[];
  auto& sm = *reinterpret_cast<DqTiles<T, D>*>(smem_raw);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), ln = lane & 31, lh = lane >> 5;

  const int hh = blockIdx.x % a.H, kvh = hh % a.Hkv, h = kvh * (a.H / a.Hkv) + hh / a.Hkv;
  const SeqTile at = ranked_tile<kPackedRows, false>(a.cu_q, a.total_q, a.cu_k, a.total_k, a.n_seqs, blockIdx.x / a.H, tiles, lane);
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
  float delta = P::dot(q, g);
  if (sizeof(T) == 2 && a.rest) {   // out's rounding would cost dq and dk half as much again as that of the weights
    P::load(g, rows_of<T>((const void*)a.rest, a.os, qbase + ic, h), lane, false);
    delta += P::dot(q, g);
  }
  g = q;
  P::load(q, rows_of<T>(a.q, a.qs, qbase + ic, h), lane, a.scale < 0.f);
  const int64_t stat = (int64_t)h * a.total_q + qbase + ic;
  const float lse = a.lse[stat] * kLog2e;
  if (i < nq) a.stats[stat + (lh ? (int64_t)a.H * a.total_q : 0)] = lh ? -delta : lse;
  const float sc = (a.scale == 0.f ? 1e-30f : fabsf(a.scale)) * kLog2e;

  f32x16 dq[MT];

  const T* kp = rows_of<T>(a.k, a.ks, kbase, kvh);
  const T* vp = rows_of<T>(a.v, a.vs, kbase, kvh);
  const int last_key = min(i0 + kPackedRows, nq) - 1 + off;
  const int n_tiles = last_key < 0 ? 0 : last_key / R + 1;
  auto load = [&](int t) {
    L::template load<W>(sm.k[t % kBuffers], kp, a.ks[0], t * R, nk - 1, wave, lane);
    L::template load<W>(sm.v[t % kBuffers], vp, a.vs[0], t * R, nk - 1, wave, lane);
  };
  bool odd = false;
  auto sums = [&](int t, auto by_rows) {
    const int t0 = t * R;
    const bool mask = t0 + R - 1 > q0 + off;   // some query of the wave does not see the whole tile
    const T *kt = sm.k[t % kBuffers], *vt = sm.v[t % kBuffers];
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      const f32x16 s = P::scores(kt + 32 * n * D, q, lane), dp = P::scores(vt + 32 * n * D, g, lane);
      float ds[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) ds[r] = __builtin_amdgcn_exp2f(fmaf(s[r], sc, -lse)) * (dp[r] - delta);
      if (mask) {
#pragma unroll
        for (int r = 0; r < 16; ++r) ds[r] = t0 + 32 * n + 8 * (r / 4) + 4 * lh + r % 4 > seen ? 0.f : ds[r];
      }
      const typename P::Weights w = P::weights(ds);
      if (by_rows && mask && L::odd(kt + 32 * n * D, lane)) P::product_by_rows(dq, kt + 32 * n * D, w, 0, seen + 1 - t0 - 32 * n, lane);
      else P::product(dq, kt + 32 * n * D, w, lane);
      if (!by_rows && mask) odd = odd || L::odd(kt + 32 * n * D, lane);
    }
  };
  auto pass = [&](auto by_rows) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) dq[mt][r] = 0.f;
    for (int t = 0; t < kBuffers - 1; ++t)
      if (t < n_tiles) load(t);
    for (int t = 0; t < n_tiles; ++t) {
      if (t + 1 < n_tiles) loads_left<2 * L::loads(W)>();
      else loads_left<0>();
      lds_barrier();   // tile t is there, and nobody reads tile t - 1 any more
      if (t + kBuffers - 1 < n_tiles) load(t + kBuffers - 1);
      if (t * R <= min(q0 + 31, nq - 1) + off) sums(t, by_rows);   // else nothing for this wave
    }
    lds_barrier();   // every wave is done with the tiles
  };
  pass(std::false_type{});
  if (any_wave(&sm.flag, odd)) pass(std::true_type{});
  if (q0 < nq)
    put_rows<T, D>(dq, a.scale, reinterpret_cast<T*>(smem_raw) + wave * 32 * kPutRow<T, D>, rows_of<T>(a.dq, a.dqs, qbase + q0, h), a.dqs[0],
                   min(32, nq - q0), lane);
}

template <typename T, int D> __global__ __launch_bounds__((kPackedThreads * kStreams<T, D>), (kWaves<T, D>)) void packed_dkdv_kernel(PackedArgs a, int tiles) {
  using P = Products<T, D>;
  constexpr int R = kQueryTile<T, D>, MT = D / 32, W = kPackedThreads / 64;
  using L = Tile<T, D, R>;
  extern __shared__ __align__(256) unsigned char smem_raw[];
  constexpr int S = kStreams<T, D>;
  auto& all = *reinterpret_cast<KeyTiles<T, D>*>(smem_raw);
  const int stream = __builtin_amdgcn_readfirstlane(threadIdx.x / kPackedThreads);
  auto& sm = all.stream[stream];
  const int tid = threadIdx.x % kPackedThreads, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), ln = lane & 31, lh = lane >> 5;

  const int kvh = blockIdx.x % a.Hkv;
  const SeqTile at = ranked_tile<kPackedRows, true>(a.cu_k, a.total_k, a.cu_q, a.total_q, a.n_seqs, blockIdx.x / a.Hkv, tiles, lane);
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
  T* const own_v = all.v + (kValuesInLds<T, D> ? wave * 32 * D : 0);
  if constexpr (kValuesInLds<T, D>)
    if (stream == 0) P::to_lds(v, own_v, lane);   // read behind the first barrier
  const float sc = (a.scale == 0.f ? 1e-30f : fabsf(a.scale)) * kLog2e;

  f32x16 dk[MT], dv[MT];

  // the tiles of queries that see any of the workgroup's keys, for every head of the group in turn
  const int first_tile = max(j0 - off, 0) / R;
  const int per_head = nq == 0 ? 0 : (nq - 1) / R + 1 - first_tile, G = a.H / a.Hkv, total = max(per_head, 0) * G;
  // the stream's n-th tile, queries `t` R .. of head `g` of the group; its next one
  struct Place { int g, t; };
  auto next = [&](Place& p) {
    for (p.t += S; p.t - first_tile >= per_head; p.t -= per_head) ++p.g;
  };
  auto load = [&](const Place& p, int n) {
    const int h = kvh * G + p.g, t0 = p.t * R, to = n % kBuffers;
    L::template load<W>(sm.q[to], rows_of<T>(a.q, a.qs, qbase, h), a.qs[0], t0, nq - 1, wave, lane);
    L::template load<W>(sm.g[to], rows_of<T>(a.dout, a.gs, qbase, h), a.gs[0], t0, nq - 1, wave, lane);
    // one word a lane: what is left of a wave, or the other statistic; every wave brings the same
#pragma unroll
    for (int x = 0; x < R / 32; ++x) {
      const int64_t at_stat = (int64_t)(R == 64 ? x : lane / 32) * a.H * a.total_q + (int64_t)h * a.total_q + qbase + min(t0 + lane % R, nq - 1);
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(a.stats + at_stat),
                                       (__attribute__((address_space(3))) void*)(sm.stats[to] + 64 * x), 4, 0, 0);
    }
  };
  constexpr int LOADS = 2 * L::loads(W) + R / 32;
  bool odd = false;
  // 32 of the queries of the stream's n-th tile, from t0 on
  auto sums = [&](int n, int part, int t0, auto by_rows) {
    // some query does not see all of the wave's keys, or is none
    const bool mask = t0 + 32 > nq || t0 < min(k0 + 31, nk - 1) - off;
    const T *qt = sm.q[n % kBuffers] + 32 * part * D, *gt = sm.g[n % kBuffers] + 32 * part * D;
    const float* stats = sm.stats[n % kBuffers] + 32 * part + 4 * lh;
    const int lo = from - t0, hi = nq - t0;   // rows that see this lane's key
    auto hidden = [&](int r) { return 8 * (r / 4) + 4 * lh + r % 4 < lo || 8 * (r / 4) + 4 * lh + r % 4 >= hi; };
    float p[16], ds[16];
    const f32x16 s = P::scores(qt, k, lane);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4_t l4 = *reinterpret_cast<const f32x4_t*>(stats + 8 * g);
#pragma unroll
      for (int e = 0; e < 4; ++e) p[4 * g + e] = __builtin_amdgcn_exp2f(fmaf(s[4 * g + e], sc, -l4[e]));
    }
    if (mask) {
#pragma unroll
      for (int r = 0; r < 16; ++r) p[r] = hidden(r) ? 0.f : p[r];
    }
    const typename P::Weights wp = P::weights(p);
    if (by_rows && mask && L::odd(gt, lane)) P::product_by_rows(dv, gt, wp, lo, hi, lane);
    else P::product(dv, gt, wp, lane);
    f32x16 dp;   // the sums start from -delta
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4_t d4 = *reinterpret_cast<const f32x4_t*>(stats + R + 8 * g);
#pragma unroll
      for (int e = 0; e < 4; ++e) dp[4 * g + e] = d4[e];
    }
    if constexpr (kValuesInLds<T, D>) dp = P::scores_lds(gt, own_v, lane, dp);
    else dp = P::scores(gt, v, lane, dp);
#pragma unroll
    for (int r = 0; r < 16; ++r) ds[r] = p[r] * dp[r];
    if (mask) {
#pragma unroll
      for (int r = 0; r < 16; ++r) ds[r] = hidden(r) ? 0.f : ds[r];
    }
    const typename P::Weights wd = P::weights(ds);
    if (by_rows && mask && L::odd(qt, lane)) P::product_by_rows(dk, qt, wd, lo, hi, lane);
    else P::product(dk, qt, wd, lane);
    if (!by_rows && mask) odd = odd || L::odd(qt, lane) || L::odd(gt, lane);
  };
  auto pass = [&](auto by_rows) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) dk[mt][r] = dv[mt][r] = 0.f;
    if (total == 0) return;
    Place now{0, first_tile - S + stream}, ahead = now;
    next(now);
    for (int n = 0; n < kBuffers - 1; ++n) {
      next(ahead);
      if (stream + S * n < total) load(ahead, n);
    }
    for (int it = stream, n = 0; it - stream < total; it += S, ++n, next(now)) {   // the streams meet at every barrier
      if (it + S < total) loads_left<LOADS>();
      else loads_left<0>();
      lds_barrier();   // tile n is there, and nobody reads tile n - 1 any more
      next(ahead);
      if (it + (kBuffers - 1) * S < total) load(ahead, n + kBuffers - 1);
      const int t0 = now.t * R;
      // else no tile, no key, or none that a query of the tile sees
#pragma unroll
      for (int x = 0; x < R / 32; ++x)
        if (it < total && k0 < nk && t0 + 32 * x + 31 >= k0 - off && t0 + 32 * x < nq) sums(n, x, t0 + 32 * x, by_rows);
    }
    lds_barrier();   // every wave is done with the tiles
  };
  pass(std::false_type{});
  if (any_wave(&all.flag, odd)) pass(std::true_type{});
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
    T* own = reinterpret_cast<T*>(smem_raw) + wave * 32 * kPutRow<T, D>;
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
