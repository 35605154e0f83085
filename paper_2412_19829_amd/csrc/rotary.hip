// Rotary positions (rotary.hpp).  A thread holds the cosines and sines of one row's pairs in two pieces of 16 bytes and walks heads with
// them, so that the angles, which take 64 bits, are taken once for several heads.  Memory bounds it.
#include "rotary.hpp"

#include "mfma.hpp"
#include "packed.hpp"

#include <algorithm>

namespace gformer {
namespace {

constexpr int kRotaryThreads = 256;
constexpr int kRotaryHeads = 8;      // heads that a thread walks

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

template <typename T> __global__ __launch_bounds__(kRotaryThreads) void rotary_kernel(RotaryArgs a) {
  using P = Piece<T>;
  constexpr int N = P::N;
  const int units = a.d / (2 * N), rows = kRotaryThreads / units;      // two pieces each
  const int tid = threadIdx.x, unit = tid % units;
  const int heads = a.H + a.Hkv, sets = (heads + kRotaryHeads - 1) / kRotaryHeads;
  const int64_t row = (int64_t)(blockIdx.x / sets) * rows + tid / units;
  const int first = blockIdx.x % sets * kRotaryHeads, last = min(first + kRotaryHeads, heads);
  if (row >= a.total) return;
  bool real = true;
  int position;
  if (a.positions) {
    position = a.positions[row];
  } else {
    // the last sequence that starts at or before the row
    int lo = 0, hi = a.n_seqs + 1;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (packed_row(a.cu, mid, a.total) <= row) lo = mid; else hi = mid;
    }
    real = lo < a.n_seqs && packed_row(a.cu, lo, a.total) <= row;
    position = (int)((uint32_t)row - (uint32_t)packed_row(a.cu, lo, a.total) + (uint32_t)(real && a.start ? a.start[lo] : 0));
  }
  if (!real && !a.zero_tail) return;

  // turning channels: the first rot / (2 N) units, two pieces that belong together each
  const bool turns = unit * 2 * N < a.rot;
  int c0 = unit * 2 * N, c1 = c0 + N;
  if (turns && !a.interleaved) {
    c0 = unit * N;
    c1 = a.rot / 2 + c0;
  }
  float c[N], s[N];
  if (turns && real) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      turn(position, a.freqs[unit * N + i], c[i], s[i]);
      c[i] *= a.factor;
      s[i] *= a.inverse ? -a.factor : a.factor;
    }
  }
  for (int h = first; h < last; ++h) {
    const bool key = h >= a.H;
    if (!turns && real && (key ? a.k == a.k_out : a.q == a.q_out)) continue;   // in place: there already
    const T* in = key ? rows_of<T>(a.k, a.ks, row, h - a.H) : rows_of<T>(a.q, a.qs, row, h);
    T* out = key ? rows_of<T>(a.k_out, a.kos, row, h - a.H) : rows_of<T>(a.q_out, a.qos, row, h);
    P x, y;
    if (!real) {
      x.w = y.w = u32x4{0, 0, 0, 0};
    } else {
      x.w = *reinterpret_cast<const u32x4*>(in + c0);
      y.w = *reinterpret_cast<const u32x4*>(in + c1);
      if (turns) {
        float u[N], v[N];
        if (a.interleaved) {
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const float p = i < N / 2 ? x.at(2 * i) : y.at(2 * i - N), q = i < N / 2 ? x.at(2 * i + 1) : y.at(2 * i + 1 - N);
            const float p2 = fmaf(p, c[i], -(q * s[i])), q2 = fmaf(q, c[i], p * s[i]);
            if (i < N / 2) {
              u[2 * i] = p2;
              u[2 * i + 1] = q2;
            } else {
              v[2 * i - N] = p2;
              v[2 * i + 1 - N] = q2;
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const float p = x.at(i), q = y.at(i);
            u[i] = fmaf(p, c[i], -(q * s[i]));
            v[i] = fmaf(q, c[i], p * s[i]);
          }
        }
        x.set(u);
        y.set(v);
      }
    }
    *reinterpret_cast<u32x4*>(out + c0) = x.w;
    *reinterpret_cast<u32x4*>(out + c1) = y.w;
  }
}

int64_t groups(int total, int H, int Hkv, int d, int n) {
  const int rows = kRotaryThreads / (d / (2 * n)), sets = (H + Hkv + kRotaryHeads - 1) / kRotaryHeads;
  return ((int64_t)total + rows - 1) / rows * sets;
}

}  // namespace

bool rotary_fits(int total, int H, int Hkv, int d) { return groups(total, H, Hkv, d, Piece<float>::N) <= most_workgroups(kRotaryThreads); }

hipError_t launch_rotary(const RotaryArgs& a, bool bf16, hipStream_t s) {
  if (bf16) rotary_kernel<uint16_t><<<dim3((unsigned)groups(a.total, a.H, a.Hkv, a.d, 8)), dim3(kRotaryThreads), 0, s>>>(a);
  else rotary_kernel<float><<<dim3((unsigned)groups(a.total, a.H, a.Hkv, a.d, 4)), dim3(kRotaryThreads), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace gformer
