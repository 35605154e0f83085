// Forward pass of attention over packed sequences (packed.hpp has the formulas): softmax in one pass over the keys, with a
// running maximum and sum per query.
//
// A workgroup holds up to 128 queries of one head, 32 a wave, and streams key and value tiles through two LDS buffers: the
// next tile's rows arrive while the present one is used.  In calls of few rows it holds 32 queries, whose waves take every
// fourth tile, each with one buffer of its own and no barrier.
//
// Bound by the matrix units and the vector work between the products of a tile (exponentials, the maximum, packing of the weights):
// 8192 tokens, 32 / 8 heads, d = 128, bf16 558 us (615 in the mean of 40 passes, whose clocks differ), 0.9 to 1.0 PFLOP/s where a plain
// product of 8192 x 8192 matrices reaches 1.32; the matrix units are busy 49 % of the time, the waves wait 24 %, LDS conflicts 1 % of its
// cycles.  The bf16 kernels of one stream keep 8 and 9 registers in memory, in the second loop (row by row) alone.  fp32, 4096 tokens, 32 / 8 heads, d = 64:
// 577 us, 119 TFLOP/s of 154.  Two blocks of 32 queries a wave halve the reads of LDS and cost a workgroup (d = 64, 49 -> 66 us);
// raised wave priorities around the products cost 7 %.
#include "packed.hpp"

#include <algorithm>

namespace gformer {
namespace {

// One stream where there are workgroups enough, else a few rows a workgroup and its waves on different keys: four of them, or two
// (fp32, d = 128 only, whose four take a compute unit's LDS).
template <typename T, int D, int STREAMS> struct FwdShape_;
template <typename T, int D> struct FwdShape_<T, D, 1> {
  using type = Shape<4, 1, sizeof(T) == 2 ? 64 : 32, 2, sizeof(T) == 4 && D == 128 ? 1 : D == 64 ? 3 : 2>;
};
template <typename T, int D> struct FwdShape_<T, D, 2> {
  using type = Shape<2, 2, 32, 2, 1>;
};
template <typename T, int D> struct FwdShape_<T, D, 4> {
  using type = Shape<1, 4, 32, 1, sizeof(T) == 4 && D == 128 ? 1 : 2>;
};
template <typename T, int D, typename F> struct alignas(kLdsAlign) FwdTiles {
  struct { alignas(kTileAlign<T, D>) T k[F::BUF][F::R * D], v[F::BUF][F::R * D]; } stream[F::S];
  int flag;
};

template <typename T, int D, typename F> __global__ __launch_bounds__(F::THREADS, F::PER_SIMD) void packed_fwd_kernel(PackedArgs a, int tiles) {
  using P = Products<T, D>;
  constexpr int R = F::R, S = F::S, ROWS = F::ROWS, NS = R / 32, MT = D / 32, W = F::RW;
  using L = Tile<T, D, R>;
  extern __shared__ __align__(kLdsAlign) unsigned char smem_raw[];
  static_assert(F::R * D * sizeof(T) % kTileAlign<T, D> == 0, "the tiles behind the first");
  auto& all = *reinterpret_cast<FwdTiles<T, D, F>*>(smem_raw);
  const int tid = threadIdx.x, lane = tid & 63, ln = lane & 31, lh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64 % W), stream = __builtin_amdgcn_readfirstlane(tid / 64 / W);
  auto& sm = all.stream[stream];

  // Heads fastest, the heads that share keys Hkv apart: workgroups are dealt to the 8 XCDs in turn, so that those of one key
  // head meet in few of them.
  const int hh = blockIdx.x % a.H, kvh = hh % a.Hkv, h = kvh * (a.H / a.Hkv) + hh / a.Hkv;
  const SeqTile at = ranked_tile<ROWS, false>(a.cu_q, a.total_q, a.cu_k, a.total_k, a.n_seqs, blockIdx.x / a.H, tiles, lane);
  if (at.first < 0) return;
  const int qbase = packed_row(a.cu_q, at.seq, a.total_q), i0 = at.first;
  if (at.seq == a.n_seqs) {
    if (a.zero_tail && i0 < a.total_q - qbase)
      zero_rows<T, D>(rows_of<T>(a.out, a.os, qbase + i0, h), a.os[0], min(ROWS, a.total_q - qbase - i0), tid, F::THREADS);
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
  // base-2 exponents are score * sc, the scale's sign is in q
  const float sc = base2_scale(a.scale);

  f32x16 o[MT];
  float m, l;   // running maximum (base 2) and this half's share of the sum

  const T* kp = rows_of<T>(a.k, a.ks, kbase, kvh);
  const T* vp = rows_of<T>(a.v, a.vs, kbase, kvh);
  const int last_key = min(i0 + ROWS, nq) - 1 + off;   // of the workgroup; < 0: no query sees any
  const int n_tiles = last_key < 0 ? 0 : last_key / R + 1;
  // tile t, the stream's n-th
  auto load_keys = [&](int t, int n) { L::template load<W>(sm.k[n % F::BUF], kp, a.ks[0], t * R, nk - 1, wave, lane); };
  auto load_values = [&](int t, int n) { L::template load<W>(sm.v[n % F::BUF], vp, a.vs[0], t * R, nk - 1, wave, lane); };
  // One buffer: the wave's own, whose next keys arrive while it weights the values, and the other way round.
  constexpr bool OWN = F::BUF == 1;
  static_assert(!OWN || W == 1);
  bool odd = false;
  auto attend = [&](int t, int nth, auto by_rows) {
    const int t0 = t * R;
    const bool mask = t0 + R - 1 > q0 + off;   // some query of the wave does not see the whole tile
    const T *kt = sm.k[nth % F::BUF], *vt = sm.v[nth % F::BUF];
    f32x16 s[NS];
    if (OWN) loads_left<L::loads(W)>();
#pragma unroll
    for (int n = 0; n < NS; ++n) s[n] = P::scores(kt + 32 * n * D, q, lane);
    if (OWN && t + S < n_tiles) {
      tile_read();
      load_keys(t + S, nth + 1);
    }
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
    if (OWN) {
      if (t + S < n_tiles) loads_left<L::loads(W)>();
      else loads_left<0>();
    }
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
    if (OWN && t + S < n_tiles) {
      tile_read();
      load_values(t + S, nth + 1);
    }
  };
  auto pass = [&](auto by_rows) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[mt][r] = 0.f;
    m = -INFINITY;
    l = 0.f;
    if (stream < n_tiles) {
      load_keys(stream, 0);
      load_values(stream, 0);
    }
    if constexpr (OWN) {
      for (int t = stream; t < n_tiles; t += S) attend(t, 0, by_rows);
    } else {
      for (int t = stream, n = 0; t - stream < n_tiles; t += S, ++n) {   // the streams meet at every barrier
        loads_left<0>();
        lds_barrier();   // tile n is there, and nobody reads tile n - 1 any more
        if (t + S < n_tiles) {
          load_keys(t + S, n + 1);
          load_values(t + S, n + 1);
        }
        if (t < n_tiles && t * R <= min(q0 + 31, nq - 1) + off) attend(t, n, by_rows);   // else nothing for this wave
      }
    }
    lds_barrier();   // every wave is done with the tiles
  };
  pass(std::false_type{});
  if (any_wave(&all.flag, odd)) pass(std::true_type{});
  if constexpr (S > 1) {
    // a lane's share of its query from every stream: the maximum, the sum and the registers of weighted values
    float* at_join = reinterpret_cast<float*>(smem_raw) + lane;
    auto slot = [&](int s, int r) -> float& { return at_join[64 * (((s - 1) * W + wave) * (16 * MT + 2) + r)]; };
    static_assert(sizeof(FwdTiles<T, D, F>) >= (S - 1) * W * 64 * (16 * MT + 2) * sizeof(float));
    if (stream) {
      slot(stream, 0) = m;
      slot(stream, 1) = l;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int r = 0; r < 16; ++r) slot(stream, 2 + 16 * mt + r) = o[mt][r];
    }
    lds_barrier();
    if (!stream) {
      float up = m;
#pragma unroll
      for (int s = 1; s < S; ++s) up = fmaxf(up, slot(s, 0));
      const float ref = up == -INFINITY ? 0.f : up, by = __builtin_amdgcn_exp2f(m - ref);
      l *= by;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[mt][r] *= by;
#pragma unroll
      for (int s = 1; s < S; ++s) {
        const float by = __builtin_amdgcn_exp2f(slot(s, 0) - ref);
        l = fmaf(slot(s, 1), by, l);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[mt][r] = fmaf(slot(s, 2 + 16 * mt + r), by, o[mt][r]);
      }
      m = up;
    }
    lds_barrier();   // the rows leave through the same memory
    if (stream) return;
  }
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

template <typename T, int D, int STREAMS> hipError_t launch(const PackedArgs& a, hipStream_t s) {
  using F = typename FwdShape_<T, D, STREAMS>::type;
  constexpr size_t smem = std::max(sizeof(FwdTiles<T, D, F>), F::ROWS * kPutRow<T, D> * sizeof(T));   // the rows leave through it
  auto kern = packed_fwd_kernel<T, D, F>;
  if (hipError_t e = allow_lds(kern, smem); e != hipSuccess) return e;
  static_assert(F::ROWS == query_rows(STREAMS) && F::THREADS == kQueryThreads);
  const int64_t tiles = packed_tiles(a.total_q, a.n_seqs, F::ROWS);
  kern<<<dim3((unsigned)(tiles * a.H)), dim3(F::THREADS), smem, s>>>(a, (int)tiles);
  return hipGetLastError();
}
// us, one stream / two / four (rows x heads): bf16, d = 64: 2048 x 8 35 / - / 19, 2048 x 16 37 / - / 24, 4096 x 16 67 / - / 65, 4000 x 12 67 / - / 52,
// 2048 x 32 38 / - / 39, 8 of 200 x 16 10 / - / 12; d = 128: 512 x 8 17 / - / 12, 2048 x 8 50 / - / 27, 512 x 32 18 / - / 13, 2048 x 16 52 / - / 41,
// 4000 x 12 95 / - / 90, 4096 x 16 101 / - / 120; fp32, d = 64: 2048 x 8 157 / - / 63, 2048 x 16 162 / - / 98, 4096 x 16 415 / - / 317, 4096 x 32 578 / - / 577;
// d = 128: 1024 x 16 - / 85 / 65, 2048 x 8 - / 161 / 106, 2048 x 16 300 / 178 / 209, 4000 x 12 570 / 523 / 548, 4096 x 16 633 / 650 / -.
template <typename T, int D> hipError_t launch(const PackedArgs& a, hipStream_t s) {
  switch (packed_streams(sizeof(T) == 4, D, a.total_q, a.H, a.n_seqs)) {
    case 1: return launch<T, D, 1>(a, s);
    case 2: if constexpr (sizeof(T) == 4 && D == 128) return launch<T, D, 2>(a, s);
    default: return launch<T, D, 4>(a, s);
  }
}

}  // namespace

// Streams divide the longest workgroup's time, and load every streamed row as many times more often.  Four of them leave room for
// two workgroups on a compute unit (fp32, d = 128: one), so up to two rounds of the unsplit workgroups are better split; at
// d = 128, whose values cost more to join, one and a half; a quarter of that where sequences are short (a mean of less than
// 512 rows) and the joins weigh more.  The mean is what the host knows, and single tokens beside a long prompt lower it: 2048 rows of 8
// heads take 28 us at d = 128 and 18 at d = 64, with 31 single tokens 55 and 39 (backward 79 and 52, 153 and 96).
int packed_streams(bool fp32, int d, int total_q, int H, int n_seqs) {
  const int units = device_compute_units();
  const int64_t workgroups = (int64_t)total_q * H / kPackedRows, most = units * (d == 64 ? 4 : 3) / 2;
  if (workgroups > (total_q < (int64_t)512 * n_seqs ? most / 4 : most)) return 1;
  return fp32 && d == 128 && workgroups > units / 2 ? 2 : 4;
}

bool packed_queries_fit(bool fp32, int d, int total_q, int H, int n_seqs) {
  return packed_tiles(total_q, n_seqs, query_rows(packed_streams(fp32, d, total_q, H, n_seqs))) * H <= most_workgroups(kQueryThreads);
}

hipError_t launch_packed_fwd(const PackedArgs& a, bool bf16, hipStream_t s) {
  if (bf16) return a.d == 128 ? launch<uint16_t, 128>(a, s) : launch<uint16_t, 64>(a, s);
  return a.d == 128 ? launch<float, 128>(a, s) : launch<float, 64>(a, s);
}

}  // namespace gformer
