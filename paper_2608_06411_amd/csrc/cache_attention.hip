// Attention of new rows over their sequences' cached keys and values.
//
//   out = sum_j p_j v_j / sum_j p_j,  p_j = 2^(c2 <q, k_j> - m),  over the tokens
//   the row sees; c2 = scale log2(e), m the running maximum (one pass).
//
// A workgroup takes one row and head; its four waves take 64 tokens each in
// turn, a token a lane for the scores and two values a lane for the sum, and
// join their (m, l, o) at the end.
#include "cache_pages.h"

namespace mapk {

namespace {

constexpr int NT = 256;

template <int DH, bool FP4>
__global__ __launch_bounds__(NT) void cache_attention_kernel(const CacheAttnArgs a) {
  __shared__ float qs[DH], os[4][DH], ms[4], ls[4];
  __shared__ float ps[4][64];
  __shared__ long long rs[4][64];
  const int b = blockIdx.z, h = blockIdx.y, i = blockIdx.x, r0 = a.off[b], n = a.off[b + 1] - r0;
  if (i >= n) return;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, kvh = h / a.G;
  const int len = cache_len(a.c, b), me = len - n + i;
  if (threadIdx.x < DH)
    qs[threadIdx.x] = bf16_to_f32(static_cast<const bf16_t*>(a.q)[(r0 + i) * a.ldq + h * DH + threadIdx.x]);
  __syncthreads();
  float m = -3.0e38f, l = 0.0f, o0 = 0.0f, o1 = 0.0f;
  for (int j0 = 64 * wave; j0 <= me; j0 += 256) {
    const int j = j0 + lane;
    const bool see = j <= me && (a.window == 0 || me - j < a.window || j < a.sinks);
    const int page = see ? cache_page(a.c, b, j) : -1;
    const long long row = page >= 0 ? cache_row(a.c, page, kvh, j) : -1;
    float z = -INFINITY;
    if (row >= 0) {
      float sum = 0.0f;
      for (int d = 0; d < DH; d += 8) {
        union { uint4 u; bf16_t e[8]; } k;
        if constexpr (FP4)
          k.u = fp4_eight(static_cast<const uint32_t*>(a.c.k)[row * (DH / 8) + d / 8], fp4_scale(a.c.ks[row * (DH / 32) + d / 32]));
        else
          k.u = *reinterpret_cast<const uint4*>(static_cast<const bf16_t*>(a.c.k) + row * DH + d);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fmaf(qs[d + e], bf16_to_f32(k.e[e]), sum);
      }
      z = sum * a.c2;
    }
    float mx = z;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off, 64));
    const float mn = fmaxf(m, mx), al = exp2f(m - mn);
    m = mn;
    const float p = row >= 0 ? exp2f(z - m) : 0.0f;
    l = l * al + p;
    o0 *= al;
    o1 *= al;
    ps[wave][lane] = p;
    rs[wave][lane] = row;
    for (int t = 0; t < 64; ++t) {
      const long long vr = rs[wave][t];
      if (vr < 0) continue;
      const float pt = ps[wave][t];
      if (DH == 64 && lane >= 32) continue;
      uint32_t w;
      if constexpr (FP4) {
        const uint32_t byte = static_cast<const uint8_t*>(a.c.v)[vr * (DH / 2) + lane];
        w = fp4_pair<0>(byte, fp4_scale(a.c.vs[vr * (DH / 32) + lane / 16]));
      } else {
        w = reinterpret_cast<const uint32_t*>(static_cast<const bf16_t*>(a.c.v) + vr * DH)[lane];
      }
      o0 = fmaf(pt, __uint_as_float(w << 16), o0);
      o1 = fmaf(pt, __uint_as_float(w & 0xffff0000u), o1);
    }
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) l += __shfl_xor(l, off, 64);
  if (2 * lane < DH) {
    os[wave][2 * lane] = o0;
    os[wave][2 * lane + 1] = o1;
  }
  if (lane == 0) {
    ms[wave] = m;
    ls[wave] = l;
  }
  __syncthreads();
  if (threadIdx.x < DH) {
    const float mm = fmaxf(fmaxf(ms[0], ms[1]), fmaxf(ms[2], ms[3]));
    float o = 0.0f, sum = 0.0f;
    for (int w = 0; w < 4; ++w) {
      const float f = exp2f(ms[w] - mm);
      o = fmaf(f, os[w][threadIdx.x], o);
      sum = fmaf(f, ls[w], sum);
    }
    static_cast<bf16_t*>(a.out)[(r0 + i) * a.ldo + h * DH + threadIdx.x] = f32_to_bf16(sum == 0.0f ? 0.0f : o / sum);
  }
}

}  // namespace

hipError_t launch_cache_attention(CacheAttnArgs& a, hipStream_t s) {
  int most = 0;
  for (int b = 0; b < a.B; ++b) most = max(most, a.off[b + 1] - a.off[b]);
  const dim3 grid(most, a.Hq, a.B), block(NT);
  if (a.fp4)
    return a.Dh == 128 ? launch_kernel("cache_attention", cache_attention_kernel<128, true>, grid, block, 0, s, a)
                       : launch_kernel("cache_attention", cache_attention_kernel<64, true>, grid, block, 0, s, a);
  return a.Dh == 128 ? launch_kernel("cache_attention", cache_attention_kernel<128, false>, grid, block, 0, s, a)
                     : launch_kernel("cache_attention", cache_attention_kernel<64, false>, grid, block, 0, s, a);
}

}  // namespace mapk
