// Norms of the query and key heads and their rotation by position, one pass.
//
//   y = x / sqrt(mean(x^2) + eps) * g,  per head of head_dim values;
//   pair i, (i, i + rot/2):  (a, b) -> (a cos t - b sin t, b cos t + a sin t),
//   t = pos[axis(i)][r] theta^(-2i/rot).
//
// A row's heads all turn by the same rot/2 angles, so a wave takes a row (or
// a share of its heads), forms one pair's sine and cosine a lane and passes
// them round through LDS.  head_dim / 16 lanes hold a head, each the two
// 16-byte pieces whose values pair up: norm, rotation and the store need no
// further exchange but the norm's sum.
// The angle goes through turns, in float64: pos * turns[i] minus its nearest
// whole number is exact but for the product's rounding (a turn's 2^-53 times
// the position), and the sine of the float32 rest is within a few 2^-24.
// Bound: the bytes.  37600 rows of 32 heads in bf16 (616 MB in and out): 116 us,
// 5.3 TB/s, the rate of a large copy.
#include "internal.h"

namespace mapk {

namespace {

constexpr int NT = 256;
constexpr int kWaves = NT / 64;

template <typename T> struct Piece;  // eight values
template <> struct Piece<bf16_t> {
  union { uint4 u; bf16_t e[8]; };
  __device__ __forceinline__ void load(const bf16_t* p) { u = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void store(bf16_t* p) const { *reinterpret_cast<uint4*>(p) = u; }
};
template <> struct Piece<float> {
  union { uint4 u[2]; float e[8]; };
  __device__ __forceinline__ void load(const float* p) {
    u[0] = reinterpret_cast<const uint4*>(p)[0];
    u[1] = reinterpret_cast<const uint4*>(p)[1];
  }
  __device__ __forceinline__ void store(float* p) const {
    reinterpret_cast<uint4*>(p)[0] = u[0];
    reinterpret_cast<uint4*>(p)[1] = u[1];
  }
};

template <typename T, int DH>
__global__ __launch_bounds__(NT) void qk_norm_rope_kernel(const QkRopeArgs a) {
  constexpr int LPH = DH / 16, HPW = 64 / LPH;  // lanes a head, heads a wave
  __shared__ float2 cs[kWaves][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, l = lane % LPH;
  const int item = blockIdx.x * kWaves + wave, r = item / a.parts, part = item - r * a.parts;
  const bool live = r < a.R;
  if (live && lane < a.rot / 2) {
    const double t = static_cast<double>(a.pos[a.axis[lane] * a.ldpos + r]) * a.turns[lane];
    float s, c;
    sincospif(2.0f * static_cast<float>(t - rint(t)), &s, &c);
    cs[wave][lane] = make_float2(c, s);
  }
  __syncthreads();
  if (!live) return;
  const int rl = a.rot / 16;  // lanes of a head that rotate
  const bool turn = l < rl;
  // this lane's two pieces: a pair's two sides, or two pieces that pass
  const int i0 = turn ? 8 * l : a.rot + 16 * (l - rl), i1 = turn ? i0 + a.rot / 2 : i0 + 8;
  float c[8], s[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float2 v = turn ? cs[wave][i0 + k] : make_float2(1.0f, 0.0f);
    c[k] = v.x;
    s[k] = v.y;
  }
  for (int h0 = part * HPW; h0 < a.Hq + a.Hkv; h0 += a.parts * HPW) {
    const int h = h0 + lane / LPH;
    if (h >= a.Hq + a.Hkv) continue;
    const bool isq = h < a.Hq;
    const int hh = isq ? h : h - a.Hq;
    const T* src = static_cast<const T*>(isq ? a.q : a.k) + r * (isq ? a.ldq : a.ldk) + hh * DH;
    T* dst = static_cast<T*>(isq ? a.q_out : a.k_out) + r * (isq ? a.ldqo : a.ldko) + hh * DH;
    const T* g = static_cast<const T*>(isq ? a.q_norm : a.k_norm);
    Piece<T> u, v;
    u.load(src + i0);
    v.load(src + i1);
    float x[8], y[8], ss = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      x[k] = to_f32<T>(u.e[k]);
      y[k] = to_f32<T>(v.e[k]);
      ss = fmaf(x[k], x[k], fmaf(y[k], y[k], ss));
    }
#pragma unroll
    for (int off = LPH / 2; off > 0; off >>= 1) ss += __shfl_xor(ss, off, 64);
    if (g) {
      // A sum of squares past float32's range, or under it where eps does not hide
      // that: once more, the head times a power of two.
      float eps = a.eps;
      const bool far = !(ss < 3e38f) | ((ss < 1e-30f) & (eps < 1e-36f));
      if (__any(far)) {
        const float t = far ? (ss < 1.0f ? 0x1p100f : 0x1p-70f) : 1.0f;
        eps = eps * t * t;
        ss = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          x[k] *= t;
          y[k] *= t;
          ss = fmaf(x[k], x[k], fmaf(y[k], y[k], ss));
        }
#pragma unroll
        for (int off = LPH / 2; off > 0; off >>= 1) ss += __shfl_xor(ss, off, 64);
      }
      const float inv = 1.0f / sqrtf(ss / static_cast<float>(DH) + eps);
      Piece<T> gu, gv;
      gu.load(g + i0);
      gv.load(g + i1);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        x[k] *= inv * to_f32<T>(gu.e[k]);
        y[k] *= inv * to_f32<T>(gv.e[k]);
      }
    }
    if (turn) {  // (kept apart: 0 * infinity would not pass a value through)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float p = x[k] * c[k] - y[k] * s[k];
        y[k] = y[k] * c[k] + x[k] * s[k];
        x[k] = p;
      }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      u.e[k] = from_f32<T>(x[k]);
      v.e[k] = from_f32<T>(y[k]);
    }
    u.store(dst + i0);
    v.store(dst + i1);
  }
}

}  // namespace

hipError_t launch_qk_norm_rope(map_dtype dt, QkRopeArgs& a, hipStream_t s) {
  const int per_wave = 64 / (a.Dh / 16), chunks = (a.Hq + a.Hkv + per_wave - 1) / per_wave;
  // A wave takes a whole row's heads, so that its angles are formed once; with few
  // rows, a share of them, so that there are about 2048 waves (224 rows of 64 heads in
  // float32: 10.7 us with a wave a row, 5.6 so).
  a.parts = static_cast<int>(max(1LL, min((long long)chunks, 2048LL / a.R)));
  const long long waves = (long long)a.R * a.parts;
  const dim3 grid(static_cast<unsigned>((waves + kWaves - 1) / kWaves));
  if (dt == MAP_BF16)
    return a.Dh == 128 ? launch_kernel("qk_norm_rope", qk_norm_rope_kernel<bf16_t, 128>, grid, dim3(NT), 0, s, a)
                       : launch_kernel("qk_norm_rope", qk_norm_rope_kernel<bf16_t, 64>, grid, dim3(NT), 0, s, a);
  return a.Dh == 128 ? launch_kernel("qk_norm_rope", qk_norm_rope_kernel<float, 128>, grid, dim3(NT), 0, s, a)
                     : launch_kernel("qk_norm_rope", qk_norm_rope_kernel<float, 64>, grid, dim3(NT), 0, s, a);
}

}  // namespace mapk
