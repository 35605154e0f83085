// Backward pass of attention over packed sequences (packed.hpp has the formulas), in two passes that take the
// weights again from the scores and the forward pass's log-sum-exp:
//   dq      queries resident, keys and values streamed; also leaves both statistics of a query for the other pass
//   dk, dv  keys resident, the queries of every head that shares them streamed, one head after another: their sums
//           need no atomics, and come out in one order
// The gradients of the scores are rounded to bf16 for their products, which costs dq and dk as much as their own rounding, and
// more where a row has few keys and a few weights decide.  In tiles that some rows see in part, short sequences' all, both
// parts of them go in: the value rounded, and what that took (the error of dq and dk over that of one rounding, 70 batches of 1 to 20
// sequences: 1.43 to 1.51 without, 1.05 to 1.34 with; dq and dk, dv at d = 64 66 and 94 us in place of 64 and 92).
// One pass for all three would save two of nine products and need atomics, whose order changes the sums.
//
// Bound like the forward pass.  4096 + 3001 + 1095 tokens, 32 / 8 heads, d = 128, bf16: dq 349 us, dk and dv 532 (373 and 593 in the mean of
// 40 passes, whose clocks differ; matrix units busy 47 and 39 %, waves waiting 31 and 44 %: dk and dv are one workgroup of eight waves on
// a compute unit there, and the longest of them takes 512 steps of 32 queries where the mean unit has 429); 8192 tokens in 8 documents, 16 heads,
// d = 64: 66 and 94; fp32, 1024 + 300 + 700 tokens, 12 heads, d = 64: 57 and 83.  What did not help: two blocks of 32 rows a wave
// (d = 64: dq 64 -> 91), three waves on a SIMD (dk, dv of the second 114 to 187 where two took 111), wave priorities (607 -> 627 and more), and all
// transposed reads of a product in one statement (d = 128 spills more: 852).
//
// As built, dk and dv do not run two tiles ahead where they have three buffers: the compiler waits for all loads at the loop's barrier,
// behind the counted wait (not in fp32 at d = 128; nor does it in dq).  The second loop, row by row, is what makes it, and at d = 128 in bf16
// also makes it keep 84 to 86 registers in memory, four of which the first loop reads back in every step; dq keeps 23 and 35 at
// d = 128, in the second loop alone.
#include "packed.hpp"

#include <algorithm>

namespace gformer {
namespace {

// waves on a SIMD that the kernels' registers are kept down for
template <typename T, int D> constexpr int kWaves = sizeof(T) == 4 && D == 128 ? 1 : 2;

// dq: as the forward pass
template <typename T, int D, int STREAMS> struct DqShape_;
template <typename T, int D> struct DqShape_<T, D, 1> {
  using type = Shape<4, 1, sizeof(T) == 2 && D == 64 ? 64 : 32, 3, sizeof(T) == 2 && D == 64 ? 3 : kWaves<T, D>>;
};
template <typename T, int D> struct DqShape_<T, D, 2> {
  using type = Shape<2, 2, 32, 2, 1>;
};
template <typename T, int D> struct DqShape_<T, D, 4> {
  using type = Shape<1, 4, 32, 1, sizeof(T) == 2 && D == 64 ? 3 : kWaves<T, D>>;
};
template <typename T, int D, typename F> struct alignas(kLdsAlign) DqTiles {
  struct { alignas(kTileAlign<T, D>) T k[F::BUF][F::R * D], v[F::BUF][F::R * D]; } stream[F::S];
  int flag;
};

// dk, dv: a causal sequence's first keys are seen by all its queries, its last by few, and there are only as many workgroups
// as key tiles and key heads.  MANY: one stream, two workgroups on a compute unit, neither of which waits for the other.  SOME: the
// longest workgroup decides, and with two streams and a compute unit of its own it takes half as long.  FEW: shorter ones yet.
enum { MANY, SOME, FEW };
int key_call(int total_k, int Hkv, int n_seqs, int groups) {
  const int units = device_compute_units();
  const bool brief = total_k < (int64_t)512 * n_seqs;   // short sequences have no long workgroups
  const int64_t workgroups = (int64_t)total_k * Hkv * groups / kPackedRows;
  if (workgroups <= (brief ? units / 2 : units)) return FEW;
  return workgroups > (brief ? units : 3 * units) ? MANY : SOME;
}
// rows and threads of a workgroup
constexpr int key_rows(int call) { return call == FEW ? 64 : kPackedRows; }
constexpr int key_threads(bool fp32, int d, int call) { return call == MANY || (fp32 && d == 128) ? 256 : 512; }
template <typename T, int D, int CALL> struct KeyShape_;
template <typename T, int D> struct KeyShape_<T, D, MANY> {
  using type = Shape<4, 1, sizeof(T) == 2 && D == 64 ? 64 : 32, sizeof(T) == 2 && D == 128 ? 2 : 3, kWaves<T, D>>;
};
template <typename T, int D> struct KeyShape_<T, D, SOME> {
  using type = Shape<4, kWaves<T, D>, sizeof(T) == 2 && D == 64 ? 64 : 32, 3, kWaves<T, D>>;
};
template <typename T, int D> struct KeyShape_<T, D, FEW> {
  using type = Shape<2, 2 * kWaves<T, D>, 32, 2, kWaves<T, D>>;
};
// its value rows stay in LDS where their registers are wanted for the sums
template <typename T, int D> constexpr bool kValuesInLds = sizeof(T) == 2 && D == 128;
template <typename T, int D, typename F> struct alignas(kLdsAlign) KeyTiles {
  struct {
    alignas(kTileAlign<T, D>) T q[F::BUF][F::R * D], g[F::BUF][F::R * D];
    float stats[F::BUF][F::R == 64 ? 128 : 64];   // in base 2: lse of the queries, then -delta
  } stream[F::S];
  alignas(kTileAlign<T, D>) T v[kValuesInLds<T, D> ? F::ROWS * D : 8];
  int flag;
};

// Adds the other streams' sums to the first one's, a register of 64 lanes at a time, through `own`: 64 MT 16 floats for each
// of their waves.
template <int S, int W, int MT> __device__ __forceinline__ void join_streams(f32x16 (&sum)[MT], float* own, int stream, int wave, int lane) {
  auto slot = [&](int s, int r) -> float& { return own[64 * (((s - 1) * W + wave) * 16 * MT + r) + lane]; };
  if (stream) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) slot(stream, 16 * mt + r) = sum[mt][r];
  }
  lds_barrier();
  if (!stream) {
#pragma unroll
    for (int s = 1; s < S; ++s)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int r = 0; r < 16; ++r) sum[mt][r] += slot(s, 16 * mt + r);
  }
  lds_barrier();
}

template <typename T, int D, typename F> __global__ __launch_bounds__(F::THREADS, F::PER_SIMD) void packed_dq_kernel(PackedArgs a, int tiles) {
  using P = Products<T, D>;
  constexpr int R = F::R, S = F::S, ROWS = F::ROWS, BUF = F::BUF, NS = R / 32, MT = D / 32, W = F::RW;
  using L = Tile<T, D, R>;
  extern __shared__ __align__(kLdsAlign) unsigned char smem_raw[];
  static_assert(F::R * D * sizeof(T) % kTileAlign<T, D> == 0, "the tiles behind the first");
  auto& all = *reinterpret_cast<DqTiles<T, D, F>*>(smem_raw);
  const int tid = threadIdx.x, lane = tid & 63, ln = lane & 31, lh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64 % W), stream = __builtin_amdgcn_readfirstlane(tid / 64 / W);
  auto& sm = all.stream[stream];

  const int hh = blockIdx.x % a.H, kvh = hh % a.Hkv, h = kvh * (a.H / a.Hkv) + hh / a.Hkv;
  const SeqTile at = ranked_tile<ROWS, false>(a.cu_q, a.total_q, a.cu_k, a.total_k, a.n_seqs, blockIdx.x / a.H, tiles, lane);
  if (at.first < 0) return;
  const int qbase = packed_row(a.cu_q, at.seq, a.total_q), i0 = at.first;
  if (at.seq == a.n_seqs) {
    if (a.zero_tail && i0 < a.total_q - qbase)
      zero_rows<T, D>(rows_of<T>(a.dq, a.dqs, qbase + i0, h), a.dqs[0], min(ROWS, a.total_q - qbase - i0), tid, F::THREADS);
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
  if (stream == 0 && i < nq) a.stats[stat + (lh ? (int64_t)a.H * a.total_q : 0)] = lh ? -delta : lse;
  const float sc = base2_scale(a.scale);

  f32x16 dq[MT];

  const T* kp = rows_of<T>(a.k, a.ks, kbase, kvh);
  const T* vp = rows_of<T>(a.v, a.vs, kbase, kvh);
  const int last_key = min(i0 + ROWS, nq) - 1 + off;
  const int n_tiles = last_key < 0 ? 0 : last_key / R + 1;
  // tile t, the stream's n-th
  auto load_keys = [&](int t, int n) { L::template load<W>(sm.k[n % BUF], kp, a.ks[0], t * R, nk - 1, wave, lane); };
  auto load_values = [&](int t, int n) { L::template load<W>(sm.v[n % BUF], vp, a.vs[0], t * R, nk - 1, wave, lane); };
  auto load = [&](int t, int n) {
    load_values(t, n);
    load_keys(t, n);
  };
  constexpr bool OWN = BUF == 1;   // as in the forward pass
  static_assert(!OWN || W == 1);
  bool odd = false;
  auto sums = [&](int t, int nth, auto by_rows) {
    const int t0 = t * R;
    const bool mask = t0 + R - 1 > q0 + off;   // some query of the wave does not see the whole tile
    const T *kt = sm.k[nth % BUF], *vt = sm.v[nth % BUF];
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      if (OWN) loads_left<L::loads(W)>();
      const f32x16 dp = P::scores(vt + 32 * n * D, g, lane);
      if (OWN && t + S < n_tiles) {
        tile_read();
        load_values(t + S, nth + 1);
        loads_left<L::loads(W)>();
      } else if (OWN) {
        loads_left<0>();
      }
      const f32x16 s = P::scores(kt + 32 * n * D, q, lane);
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
      if constexpr (sizeof(T) == 2)
        if (mask) {   // both parts of the gradients of the scores
          const typename P::Weights rest = P::rests(ds, w);
          if (by_rows && L::odd(kt + 32 * n * D, lane)) P::product_by_rows(dq, kt + 32 * n * D, rest, 0, seen + 1 - t0 - 32 * n, lane);
          else P::product(dq, kt + 32 * n * D, rest, lane);
        }
      if (!by_rows && mask) odd = odd || L::odd(kt + 32 * n * D, lane);
    }
    if (OWN && t + S < n_tiles) {
      tile_read();
      load_keys(t + S, nth + 1);
    }
  };
  auto pass = [&](auto by_rows) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) dq[mt][r] = 0.f;
    for (int n = 0; n < (OWN ? 1 : BUF - 1); ++n)
      if (stream + S * n < n_tiles) load(stream + S * n, n);
    if constexpr (OWN) {
      for (int t = stream; t < n_tiles; t += S) sums(t, 0, by_rows);
    } else {
      for (int t = stream, n = 0; t - stream < n_tiles; t += S, ++n) {   // the streams meet at every barrier
        if (BUF > 2 && t + S < n_tiles) loads_left<2 * L::loads(W)>();
        else loads_left<0>();
        lds_barrier();   // tile n is there, and nobody reads tile n - 1 any more
        if (t + (BUF - 1) * S < n_tiles) load(t + (BUF - 1) * S, n + BUF - 1);
        if (t < n_tiles && t * R <= min(q0 + 31, nq - 1) + off) sums(t, n, by_rows);   // else nothing for this wave
      }
    }
    lds_barrier();   // every wave is done with the tiles
  };
  pass(std::false_type{});
  if (any_wave(&all.flag, odd)) pass(std::true_type{});
  if constexpr (S > 1) {
    static_assert(sizeof(DqTiles<T, D, F>) >= (S - 1) * W * 64 * 16 * MT * sizeof(float));
    join_streams<S, W, MT>(dq, reinterpret_cast<float*>(smem_raw), stream, wave, lane);
    if (stream) return;
  }
  if (q0 < nq)
    put_rows<T, D>(dq, a.scale, reinterpret_cast<T*>(smem_raw) + wave * 32 * kPutRow<T, D>, rows_of<T>(a.dq, a.dqs, qbase + q0, h), a.dqs[0],
                   min(32, nq - q0), lane);
}

template <typename T, int D, typename F> __global__ __launch_bounds__(F::THREADS, F::PER_SIMD) void packed_dkdv_kernel(PackedArgs a, int tiles, int groups) {
  using P = Products<T, D>;
  constexpr int R = F::R, S = F::S, ROWS = F::ROWS, BUF = F::BUF, MT = D / 32, W = F::RW;
  using L = Tile<T, D, R>;
  extern __shared__ __align__(kLdsAlign) unsigned char smem_raw[];
  static_assert(F::R * D * sizeof(T) % kTileAlign<T, D> == 0, "the tiles behind the first");
  auto& all = *reinterpret_cast<KeyTiles<T, D, F>*>(smem_raw);
  const int tid = threadIdx.x, lane = tid & 63, ln = lane & 31, lh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64 % W), stream = __builtin_amdgcn_readfirstlane(tid / 64 / W);
  auto& sm = all.stream[stream];

  const int unit = blockIdx.x % (a.Hkv * groups), kvh = unit % a.Hkv, part = unit / a.Hkv;
  const SeqTile at = ranked_tile<ROWS, true>(a.cu_k, a.total_k, a.cu_q, a.total_q, a.n_seqs, blockIdx.x / (a.Hkv * groups), tiles, lane);
  if (at.first < 0) return;
  const int kbase = packed_row(a.cu_k, at.seq, a.total_k), j0 = at.first;
  if (at.seq == a.n_seqs) {
    if (a.zero_tail && part == 0 && j0 < a.total_k - kbase) {
      const int rows = min(ROWS, a.total_k - kbase - j0);
      zero_rows<T, D>(rows_of<T>(a.dk, a.dks, kbase + j0, kvh), a.dks[0], rows, tid, F::THREADS);
      zero_rows<T, D>(rows_of<T>(a.dv, a.dvs, kbase + j0, kvh), a.dvs[0], rows, tid, F::THREADS);
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
  const float sc = base2_scale(a.scale);

  f32x16 dk[MT], dv[MT];

  // the tiles of queries that see any of the workgroup's keys, for every head of its part of the group in turn
  const int first_tile = max(j0 - off, 0) / R;
  const int per_head = nq == 0 ? 0 : (nq - 1) / R + 1 - first_tile, G = a.H / a.Hkv / groups, total = max(per_head, 0) * G;
  // the stream's n-th tile, queries `t` R .. of head `g` of the group; its next one
  struct Place { int g, t; };
  auto next = [&](Place& p) {
    for (p.t += S; p.t - first_tile >= per_head; p.t -= per_head) ++p.g;
  };
  auto load = [&](const Place& p, int n) {
    const int h = (kvh * groups + part) * G + p.g, t0 = p.t * R, to = n % BUF;
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
    const T *qt = sm.q[n % BUF] + 32 * part * D, *gt = sm.g[n % BUF] + 32 * part * D;
    const float* stats = sm.stats[n % BUF] + 32 * part + 4 * lh;
    const int lo = from - t0, hi = nq - t0;   // rows that see this lane's key
    auto hide = [&](float (&x)[16]) {
      int first = lo - 4 * lh;
      asm volatile("" : "+v"(first));   // compared anew each time: 16 kept results would take 32 scalar registers
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = 8 * (r / 4) + r % 4 < first || 8 * (r / 4) + r % 4 >= hi - 4 * lh ? 0.f : x[r];
    };
    float p[16], ds[16];
    const f32x16 s = P::scores(qt, k, lane);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4_t l4 = *reinterpret_cast<const f32x4_t*>(stats + 8 * g);
#pragma unroll
      for (int e = 0; e < 4; ++e) p[4 * g + e] = __builtin_amdgcn_exp2f(fmaf(s[4 * g + e], sc, -l4[e]));
    }
    if (mask) hide(p);
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
    if (mask) hide(ds);
    const typename P::Weights wd = P::weights(ds);
    if (by_rows && mask && L::odd(qt, lane)) P::product_by_rows(dk, qt, wd, lo, hi, lane);
    else P::product(dk, qt, wd, lane);
    if constexpr (sizeof(T) == 2)
      if (mask) {
        const typename P::Weights rest = P::rests(ds, wd);
        if (by_rows && L::odd(qt, lane)) P::product_by_rows(dk, qt, rest, lo, hi, lane);
        else P::product(dk, qt, rest, lane);
      }
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
    for (int n = 0; n < BUF - 1; ++n) {
      next(ahead);
      if (stream + S * n < total) load(ahead, n);
    }
    for (int it = stream, n = 0; it - stream < total; it += S, ++n, next(now)) {   // the streams meet at every barrier
      if (BUF > 2 && it + S < total) loads_left<LOADS>();
      else loads_left<0>();
      lds_barrier();   // tile n is there, and nobody reads tile n - 1 any more
      next(ahead);
      if (it + (BUF - 1) * S < total) load(ahead, n + BUF - 1);
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
    static_assert(sizeof(all.stream) >= (S - 1) * W * 64 * 16 * MT * sizeof(float));
    join_streams<S, W, MT>(dk, reinterpret_cast<float*>(smem_raw), stream, wave, lane);
    join_streams<S, W, MT>(dv, reinterpret_cast<float*>(smem_raw), stream, wave, lane);
    if (stream) return;
  }
  if (k0 >= nk) return;
  if (groups > 1) {
    // this part's sums, in 32 bits
    float* own = reinterpret_cast<float*>(smem_raw) + wave * 32 * kPutRow<float, D>;
    const int64_t size = (int64_t)a.total_k * a.Hkv * D, row = (int64_t)a.Hkv * D;
    float* to = a.sums + 2 * part * size + (kbase + k0) * row + kvh * D;
    put_rows<float, D>(dk, a.scale, own, to, row, min(32, nk - k0), lane);
    put_rows<float, D>(dv, 1.f, own, to + size, row, min(32, nk - k0), lane);
  } else {
    T* own = reinterpret_cast<T*>(smem_raw) + wave * 32 * kPutRow<T, D>;
    put_rows<T, D>(dk, a.scale, own, rows_of<T>(a.dk, a.dks, kbase + k0, kvh), a.dks[0], min(32, nk - k0), lane);
    put_rows<T, D>(dv, 1.f, own, rows_of<T>(a.dv, a.dvs, kbase + k0, kvh), a.dvs[0], min(32, nk - k0), lane);
  }
}

// dk and dv of the sequences' rows from the sums of every part of the heads, four columns a thread.  Bound by memory, and small:
// the heads are parted only where there are few rows (at most 128 a compute unit, of all key heads).
template <typename T, int D> __global__ __launch_bounds__(256) void packed_add_kernel(PackedArgs a, int groups) {
  constexpr int C = D / 4;
  const int64_t unit = ((int64_t)blockIdx.x * 256 + threadIdx.x) / C;   // (row, head), dk's and then dv's
  const int64_t units = (int64_t)a.total_k * a.Hkv, at = unit % units;
  const int c = 4 * (threadIdx.x % C), head = (int)(at % a.Hkv), row = (int)(at / a.Hkv);
  if (unit >= 2 * units || row < packed_row(a.cu_k, 0, a.total_k) || row >= packed_row(a.cu_k, a.n_seqs, a.total_k)) return;
  f32x4_t x = {0.f, 0.f, 0.f, 0.f};
  for (int g = 0; g < groups; ++g) x += *reinterpret_cast<const f32x4_t*>(a.sums + (2 * g * units + unit) * D + c);
  T* to = unit < units ? rows_of<T>(a.dk, a.dks, row, head) : rows_of<T>(a.dv, a.dvs, row, head);
  Products<T, D>::put4(to + c, x[0], x[1], x[2], x[3]);
}

int64_t add_workgroups(int total_k, int Hkv, int d) { return ((int64_t)total_k * Hkv * 2 * (d / 4) + 255) / 256; }

template <typename T, int D, int STREAMS> hipError_t launch_dq(const PackedArgs& a, hipStream_t s) {
  using F = typename DqShape_<T, D, STREAMS>::type;
  static_assert(F::ROWS == query_rows(STREAMS) && F::THREADS == kQueryThreads);
  constexpr size_t smem = std::max(sizeof(DqTiles<T, D, F>), F::ROWS * kPutRow<T, D> * sizeof(T));   // the rows leave through it
  auto kern = packed_dq_kernel<T, D, F>;
  if (hipError_t e = allow_lds(kern, smem); e != hipSuccess) return e;
  const int64_t tiles = packed_tiles(a.total_q, a.n_seqs, F::ROWS);
  kern<<<dim3((unsigned)(tiles * a.H)), dim3(F::THREADS), smem, s>>>(a, (int)tiles);
  return hipGetLastError();
}
template <typename T, int D, int CALL> hipError_t launch_dkdv(const PackedArgs& a, int groups, hipStream_t s) {
  using F = typename KeyShape_<T, D, CALL>::type;
  static_assert(F::ROWS == key_rows(CALL) && F::THREADS == key_threads(sizeof(T) == 4, D, CALL));
  constexpr size_t smem = std::max(sizeof(KeyTiles<T, D, F>), F::ROWS * kPutRow<float, D> * sizeof(float));
  auto kern = packed_dkdv_kernel<T, D, F>;
  if (hipError_t e = allow_lds(kern, smem); e != hipSuccess) return e;
  const int64_t tiles = packed_tiles(a.total_k, a.n_seqs, F::ROWS);
  kern<<<dim3((unsigned)(tiles * a.Hkv * groups)), dim3(F::THREADS), smem, s>>>(a, (int)tiles, groups);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || groups == 1) return e;
  packed_add_kernel<T, D><<<dim3((unsigned)add_workgroups(a.total_k, a.Hkv, D)), dim3(256), 0, s>>>(a, groups);
  return hipGetLastError();
}
// dk, dv in two streams / one, us of the whole pass (keys x key heads): bf16, d = 64: 4 of 1000 x 32 118 / 104, 16 of 100 x 32 38 / 30, 4096 x 16 175 / 202,
// 8 of 200 x 16 34 / 36; d = 128: 4 of 1000 x 32 205 / 182, 16 of 100 x 32 61 / 49, 4096 x 16 304 / 346; fp32, d = 64: 4 of 1000 x 32 583 / 579,
// 16 of 100 x 32 103 / 88, 4096 x 16 1016 / 1213.
template <typename T, int D> hipError_t launch(const PackedArgs& a, hipStream_t s) {
  hipError_t e;
  switch (packed_streams(sizeof(T) == 4, D, a.total_q, a.H, a.n_seqs)) {
    case 1: e = launch_dq<T, D, 1>(a, s); break;
    case 2: if constexpr (sizeof(T) == 4 && D == 128) { e = launch_dq<T, D, 2>(a, s); break; }
    default: e = launch_dq<T, D, 4>(a, s);
  }
  if (e != hipSuccess || a.total_k == 0) return e;
  const int groups = packed_head_groups(a.total_k, a.H, a.Hkv);
  switch (key_call(a.total_k, a.Hkv, a.n_seqs, groups)) {
    case FEW: return launch_dkdv<T, D, FEW>(a, groups, s);
    case SOME: return launch_dkdv<T, D, SOME>(a, groups, s);
    default: return launch_dkdv<T, D, MANY>(a, groups, s);
  }
}

}  // namespace

// Where key heads are few, the workgroups that walk all query heads of one are few and long: the heads are parted until
// there is a workgroup for every compute unit.  Parts divide a group evenly; where the next number of them that does would make
// more than four for every compute unit (seven heads, say, and nearly enough rows), whose sums cost more than idle units, it is not taken.
int packed_head_groups(int total_k, int H, int Hkv) {
  const int G = H / Hkv;
  const int64_t rows = (int64_t)total_k * Hkv, enough = (int64_t)device_compute_units() * kPackedRows;
  int groups = 1;
  while (groups < G && rows * groups < enough) {
    int next = groups + 1;
    while (G % next != 0) ++next;
    if (rows * next > 4 * enough) break;
    groups = next;
  }
  return groups;
}

bool packed_keys_fit(bool fp32, int d, int total_k, int H, int Hkv, int n_seqs) {
  const int groups = packed_head_groups(total_k, H, Hkv), call = key_call(total_k, Hkv, n_seqs, groups);
  return packed_tiles(total_k, n_seqs, key_rows(call)) * Hkv * groups <= most_workgroups(key_threads(fp32, d, call)) &&
         (groups == 1 || add_workgroups(total_k, Hkv, d) <= most_workgroups(256));
}

hipError_t launch_packed_bwd(const PackedArgs& a, bool bf16, hipStream_t s) {
  if (bf16) return a.d == 128 ? launch<uint16_t, 128>(a, s) : launch<uint16_t, 64>(a, s);
  return a.d == 128 ? launch<float, 128>(a, s) : launch<float, 64>(a, s);
}

}  // namespace gformer
