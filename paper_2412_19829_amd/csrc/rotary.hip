// Rotary positions (rotary.hpp).  The angles, which take 64 bits, are taken once for all heads of a row.  Memory bounds it: 7406 rows, 7206
// of which turn, of 32 / 8 heads, d = 128, bf16 (148 MB read and written) 28.7 us, 5.1 TB/s; 4 rows of 12 / 12 heads, d = 64: 2.7, launch and trips to
// memory.  What is read need not stay in the caches, what is written is what attention reads next: over more tensors in turn 31.4 us with
// such loads and 34.5 without, with packed attention over sequences of 281 behind it 138 and 142; with such stores too 28.3, but 143 then.
#include "rotary.hpp"

#include "mfma.hpp"
#include "packed.hpp"

#include <algorithm>

namespace gformer {
namespace {

constexpr int kRotaryThreads = 256;
constexpr int kRows = 4;             // of a workgroup
constexpr int kBatch = 4;            // heads that a thread has on their way

// cos and sin of position x frequency.  The product and its remainder of quarter turns are taken in 64 bits: a far position's angle
// has lost its fraction in 32.  What is left is at most pi/4, where the series' first terms behind those taken are below 2^-28.
__device__ __forceinline__ void turn(int position, float freq, float& c, float& s) {
  const double t = (double)position * (double)freq;
  const double k = rint(t * 0.63661977236758134308);                     // 2 / pi
  const double r2 = fma(-k, 6.123233995736766036e-17, fma(-k, 1.57079632679489661923, t));   // pi / 2 in two parts
  const float r = (float)r2, z = r * r;
  float sr = fmaf(z, 2.7557319e-6f, -1.9841270e-4f);                     // 1/9!, -1/7!
  sr = fmaf(z, sr, 8.3333333e-3f);
  sr = fmaf(z, sr, -1.6666667e-1f);
  sr = fmaf(r * z, sr, r);
  float cr = fmaf(z, -2.7557319e-7f, 2.4801587e-5f);                     // -1/10!, 1/8!
  cr = fmaf(z, cr, -1.3888889e-3f);
  cr = fmaf(z, cr, 4.1666667e-2f);
  cr = fmaf(z, cr, -0.5f);
  cr = fmaf(z, cr, 1.f);
  const int quarter = (int)(k - 4.0 * floor(k * 0.25));                  // 0 to 3
  const float cs = quarter & 1 ? sr : cr, sn = quarter & 1 ? cr : sr;
  c = quarter == 1 || quarter == 2 ? -cs : cs;
  s = quarter >= 2 ? -sn : sn;
}

template <typename T> struct Piece;       // 16 bytes of a row
template <> struct Piece<uint16_t> {
  static constexpr int N = 8;
  u32x4 w;
  __device__ __forceinline__ float at(int i) const { return i % 2 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]); }
  __device__ __forceinline__ void set(const float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
  }
};
template <> struct Piece<float> {
  static constexpr int N = 4;
  u32x4 w;
  __device__ __forceinline__ float at(int i) const { return __uint_as_float(w[i]); }
  __device__ __forceinline__ void set(const float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(x[i]);
  }
};

// The last sequence that starts at or before a row (n_seqs: the row lies behind them all, -1: in front), by 64 probes at a time.
__device__ __forceinline__ int sequence_of(const int32_t* cu, int n_seqs, int total, int row, int lane) {
  int lo = 0, hi = n_seqs + 1;
  do {
    const int step = (hi - lo + 63) / 64, s = lo + lane * step;
    const int n = __popcll(__builtin_amdgcn_ballot_w64(s < hi && packed_row(cu, min(s, n_seqs), total) <= row));
    if (n == 0) return -1;
    lo = __builtin_amdgcn_readfirstlane(lo + (n - 1) * step);
    hi = __builtin_amdgcn_readfirstlane(min(hi, lo + step));
  } while (hi - lo > 1);
  return lo;
}

// A workgroup takes ROWS rows, all heads.  Its threads take the rows' angles first, one pair each, and exchange them through LDS; then a
// thread keeps one row's cosines and sines of its pieces and walks heads, kBatch of them on their way at once.
template <typename T, int D, int ROWS, bool INTERLEAVED> __global__ __launch_bounds__(kRotaryThreads) void rotary_kernel(RotaryArgs a) {
  using P = Piece<T>;
  constexpr int N = P::N, UNITS = D / (2 * N), SETS = kRotaryThreads / (UNITS * ROWS), HALF = D / 2;
  static_assert(SETS >= 1 && ROWS <= kRotaryThreads / 64, "a wave for each row's position");
  __shared__ __align__(16) float sm_c[ROWS][HALF], sm_s[ROWS][HALF];
  __shared__ int sm_position[ROWS];
  __shared__ bool sm_real[ROWS];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int unit = tid % UNITS, r = tid / UNITS % ROWS, set = tid / (UNITS * ROWS);
  const int64_t row0 = (int64_t)blockIdx.x * ROWS;
  const int half = a.rot / 2;
  const bool mine = row0 + r < a.total;

  // turning channels: the first rot / (2 N) units, two pieces that belong together each
  const bool turns = unit * 2 * N < a.rot;
  int c0 = unit * 2 * N, c1 = c0 + N;
  if (turns && !INTERLEAVED) {
    c0 = unit * N;
    c1 = half + c0;
  }
  const int heads = a.H + a.Hkv;
  auto from = [&](int h) { return h < a.H ? rows_of<T>(a.q, a.qs, row0 + r, h) : rows_of<T>(a.k, a.ks, row0 + r, h - a.H); };
  auto to = [&](int h) { return h < a.H ? rows_of<T>(a.q_out, a.qos, row0 + r, h) : rows_of<T>(a.k_out, a.kos, row0 + r, h - a.H); };
  P x[kBatch], y[kBatch];
  auto load = [&](int h0) {
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int h = h0 + j * SETS;
      if (mine && h < heads) {
        x[j].w = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(from(h) + c0));
        y[j].w = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(from(h) + c1));
      }
    }
  };
  load(set);   // on their way while the angles are taken

  // wave by wave a row's position; no sequence's row: it is zeroed or left
  if (wave < ROWS && row0 + wave < a.total) {
    const int row = (int)row0 + wave;
    int position;
    bool real = true;
    if (a.positions) {
      position = a.positions[row];
    } else {
      const int seq = sequence_of(a.cu, a.n_seqs, a.total, row, lane);
      real = seq >= 0 && seq < a.n_seqs;
      position = real ? (int)((uint32_t)row - (uint32_t)packed_row(a.cu, seq, a.total) + (uint32_t)(a.start ? a.start[seq] : 0)) : 0;
    }
    if (lane == 0) {
      sm_position[wave] = position;
      sm_real[wave] = real;
    }
  }
  lds_barrier();
  for (int i = tid; i < ROWS * half; i += kRotaryThreads) {
    if (row0 + i / half < a.total) {
      float c, s;
      turn(sm_position[i / half], a.freqs[i % half], c, s);
      sm_c[i / half][i % half] = c * a.factor;
      sm_s[i / half][i % half] = s * (a.inverse ? -a.factor : a.factor);
    }
  }
  lds_barrier();
  if (!mine) return;
  const bool real = sm_real[r];
  if (!real && !a.zero_tail) return;
  float c[N], s[N];
  if (turns) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      c[i] = sm_c[r][unit * N + i];
      s[i] = sm_s[r][unit * N + i];
    }
  }
  for (int h0 = set; h0 < heads; h0 += kBatch * SETS) {
    if (h0 != set) load(h0);
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int h = h0 + j * SETS;
      if (h >= heads) break;
      if (!real) {
        x[j].w = y[j].w = u32x4{0, 0, 0, 0};
      } else if (turns) {
        float u[N], v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const bool low = !INTERLEAVED || i < N / 2;   // the pair's two channels
          const float p = INTERLEAVED ? (low ? x[j].at(2 * i % N) : y[j].at(2 * i % N)) : x[j].at(i);
          const float q = INTERLEAVED ? (low ? x[j].at(2 * i % N + 1) : y[j].at(2 * i % N + 1)) : y[j].at(i);
          const float p2 = fmaf(p, c[i], -(q * s[i])), q2 = fmaf(q, c[i], p * s[i]);
          if (!INTERLEAVED) {
            u[i] = p2;
            v[i] = q2;
          } else if (low) {
            u[2 * i % N] = p2;
            u[2 * i % N + 1] = q2;
          } else {
            v[2 * i % N] = p2;
            v[2 * i % N + 1] = q2;
          }
        }
        x[j].set(u);
        y[j].set(v);
      } else if (h < a.H ? a.q == a.q_out : a.k == a.k_out) {
        continue;   // in place: there already
      }
      *reinterpret_cast<u32x4*>(to(h) + c0) = x[j].w;
      *reinterpret_cast<u32x4*>(to(h) + c1) = y[j].w;
    }
  }
}

// From here on, four rows for every compute unit, a workgroup takes kRows rows, below it one.  us with one and with four: 32 / 8 heads, d = 128, bf16 512
// rows 4.6 and 5.9, 1024 6.0 and 7.0, 2048 10.7 and 11.2, 4096 18.5 and 17.1; 12 / 12 heads, d = 64 1024 6.4 and 6.3, 2048 6.0 and 5.1, 4096 9.7 and 7.3.  Rows of
// many bytes would want it at about 2500.
constexpr int kManyRows = 1024;

template <typename T, int D, int ROWS> void launch(const RotaryArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(((int64_t)a.total + ROWS - 1) / ROWS));
  if (a.interleaved) rotary_kernel<T, D, ROWS, true><<<grid, dim3(kRotaryThreads), 0, s>>>(a);
  else rotary_kernel<T, D, ROWS, false><<<grid, dim3(kRotaryThreads), 0, s>>>(a);
}
template <typename T, int D> void launch(const RotaryArgs& a, hipStream_t s) {
  if (a.total >= kManyRows) launch<T, D, kRows>(a, s);
  else launch<T, D, 1>(a, s);
}

}  // namespace

bool rotary_fits(int total) { return ((int64_t)total + kRows - 1) / kRows <= most_workgroups(kRotaryThreads); }

hipError_t launch_rotary(const RotaryArgs& a, bool bf16, hipStream_t s) {
  if (bf16) a.d == 128 ? launch<uint16_t, 128>(a, s) : launch<uint16_t, 64>(a, s);
  else a.d == 128 ? launch<float, 128>(a, s) : launch<float, 64>(a, s);
  return hipGetLastError();
}

}  // namespace gformer
