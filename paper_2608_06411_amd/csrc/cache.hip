// Rows of keys and values to the pages of a cache and back.
//
// Both directions move 16 bytes (eight bf16 values) a lane.  A workgroup takes
// 16 consecutive new rows of one sequence and runs through their (head, row)
// pairs with the row fastest: the rows of a head lie next to each other in a
// page, so what a workgroup writes (reads) there at a time is contiguous, and a
// cache line of 4-bit codes or of scale bytes, which holds several tokens, is
// written by one compute unit and not by several dies' L2 caches in turn.
// Bound: the bytes, 2 rows (keys, values) read and written.
//
// 4 bits: the largest magnitude of 32 values (four lanes) has the bits of a
// bf16 number, so the smallest e with max <= 7 * 2^e is its exponent minus 2,
// one more where its seven mantissa bits pass those of 1.75 (0x60).
#include "cache_pages.h"

namespace mapk {

namespace {

constexpr int NT = 256;
constexpr int kTile = 16;  // rows

struct Eight {
  union { uint4 u; bf16_t e[8]; uint32_t w[4]; };
};

// Scale byte of 32 values whose largest magnitude has these (bf16) bits: at
// most 2^125, whose 6 is the largest level that bf16 still holds.
__device__ __forceinline__ uint32_t fp4_byte(uint32_t amax) {
  if (amax >= 0x7f80u) return 255u;
  const int e = static_cast<int>(amax >> 7) - 2 + ((amax & 0x7fu) > 0x60u ? 1 : 0);
  return static_cast<uint32_t>(min(max(e, 1), 125 + 127));
}

// The largest magnitude (as bits) of eight values.
__device__ __forceinline__ uint32_t amax_bits(const Eight& v) {
  uint32_t m = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) m = max(m, static_cast<uint32_t>(v.e[k] & 0x7fffu));
  return m;
}

__device__ __forceinline__ uint32_t fp4_codes(const Eight& v, uint32_t byte) {
  if (byte == 255u) return 0u;
  const float s = fp4_scale(byte);
  uint32_t r = 0u;  // (nearest level, ties to the even code, at most 6)
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2_t, v.w[0]), s, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2_t, v.w[1]), s, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2_t, v.w[2]), s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2_t, v.w[3]), s, 3);
}

template <int DH, bool FP4>
__global__ __launch_bounds__(NT) void cache_append_kernel(const CacheRowsArgs a) {
  constexpr int LPH = DH / 8, PAIRS = NT / LPH;  // lanes a (head, row) pair, pairs at a time
  const int b = blockIdx.z, r0 = a.off[b], n = a.off[b + 1] - r0;
  const int t0 = blockIdx.x * kTile, nt = min(kTile, n - t0);
  if (nt <= 0) return;
  const int first = cache_len(a.c, b) - n;  // token of the sequence's first row
  const int l = threadIdx.x % LPH;
  for (int it = blockIdx.y * PAIRS + threadIdx.x / LPH; it < nt * a.c.heads; it += a.parts * PAIRS) {
    const int h = it / nt, i = t0 + it - h * nt, j = first + i;
    if (j < 0) continue;
    const int page = cache_page(a.c, b, j);
    if (page < 0) continue;
    const long long row = cache_row(a.c, page, h, j);
    Eight k, v;
    k.u = *reinterpret_cast<const uint4*>(static_cast<const bf16_t*>(a.k) + (r0 + i) * a.ldk + h * DH + 8 * l);
    v.u = *reinterpret_cast<const uint4*>(static_cast<const bf16_t*>(a.v) + (r0 + i) * a.ldv + h * DH + 8 * l);
    if constexpr (!FP4) {
      *reinterpret_cast<uint4*>(static_cast<bf16_t*>(a.c.k) + row * DH + 8 * l) = k.u;
      *reinterpret_cast<uint4*>(static_cast<bf16_t*>(a.c.v) + row * DH + 8 * l) = v.u;
    } else {
      // (a pair's lanes are all here or all away: the exchange stays within them)
      uint32_t mk = amax_bits(k), mv = amax_bits(v);
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) {
        mk = max(mk, static_cast<uint32_t>(__shfl_xor(static_cast<int>(mk), o, 64)));
        mv = max(mv, static_cast<uint32_t>(__shfl_xor(static_cast<int>(mv), o, 64)));
      }
      const uint32_t bk = fp4_byte(mk), bv = fp4_byte(mv);
      static_cast<uint32_t*>(a.c.k)[row * LPH + l] = fp4_codes(k, bk);
      static_cast<uint32_t*>(a.c.v)[row * LPH + l] = fp4_codes(v, bv);
      if ((l & 3) == 0) {
        a.c.ks[row * (DH / 32) + l / 4] = static_cast<uint8_t>(bk);
        a.c.vs[row * (DH / 32) + l / 4] = static_cast<uint8_t>(bv);
      }
    }
  }
}

template <int DH, bool FP4>
__global__ __launch_bounds__(NT) void cache_read_kernel(const CacheRowsArgs a) {
  constexpr int LPH = DH / 8, PAIRS = NT / LPH;
  const int b = blockIdx.z, r0 = a.off[b], n = a.off[b + 1] - r0;
  const int t0 = blockIdx.x * kTile, nt = min(kTile, n - t0);
  if (nt <= 0) return;
  const int len = cache_len(a.c, b), l = threadIdx.x % LPH;
  for (int it = blockIdx.y * PAIRS + threadIdx.x / LPH; it < nt * a.c.heads; it += a.parts * PAIRS) {
    const int h = it / nt, i = t0 + it - h * nt, j = a.slots ? a.slots[r0 + i] : i;
    const int page = j >= 0 && j < len ? cache_page(a.c, b, j) : -1;
    Eight k, v;
    k.u = v.u = make_uint4(0u, 0u, 0u, 0u);
    if (page >= 0) {
      const long long row = cache_row(a.c, page, h, j);
      if constexpr (!FP4) {
        k.u = *reinterpret_cast<const uint4*>(static_cast<const bf16_t*>(a.c.k) + row * DH + 8 * l);
        v.u = *reinterpret_cast<const uint4*>(static_cast<const bf16_t*>(a.c.v) + row * DH + 8 * l);
      } else {
        k.u = fp4_eight(static_cast<const uint32_t*>(a.c.k)[row * LPH + l], fp4_scale(a.c.ks[row * (DH / 32) + l / 4]));
        v.u = fp4_eight(static_cast<const uint32_t*>(a.c.v)[row * LPH + l], fp4_scale(a.c.vs[row * (DH / 32) + l / 4]));
      }
    }
    *reinterpret_cast<uint4*>(static_cast<bf16_t*>(a.k) + (r0 + i) * a.ldk + h * DH + 8 * l) = k.u;
    *reinterpret_cast<uint4*>(static_cast<bf16_t*>(a.v) + (r0 + i) * a.ldv + h * DH + 8 * l) = v.u;
  }
}

// Tiles of the longest sequence, and workgroups a tile.
dim3 rows_grid(CacheRowsArgs& a) {
  int most = 0;
  for (int b = 0; b < a.B; ++b) most = max(most, a.off[b + 1] - a.off[b]);
  a.parts = 1;
  return dim3((most + kTile - 1) / kTile, a.parts, a.B);
}

}  // namespace

hipError_t launch_cache_append(CacheRowsArgs& a, hipStream_t s) {
  const dim3 grid = rows_grid(a), block(NT);
  if (a.fp4)
    return a.Dh == 128 ? launch_kernel("cache_append", cache_append_kernel<128, true>, grid, block, 0, s, a)
                       : launch_kernel("cache_append", cache_append_kernel<64, true>, grid, block, 0, s, a);
  return a.Dh == 128 ? launch_kernel("cache_append", cache_append_kernel<128, false>, grid, block, 0, s, a)
                     : launch_kernel("cache_append", cache_append_kernel<64, false>, grid, block, 0, s, a);
}

hipError_t launch_cache_read(CacheRowsArgs& a, hipStream_t s) {
  const dim3 grid = rows_grid(a), block(NT);
  if (a.fp4)
    return a.Dh == 128 ? launch_kernel("cache_read", cache_read_kernel<128, true>, grid, block, 0, s, a)
                       : launch_kernel("cache_read", cache_read_kernel<64, true>, grid, block, 0, s, a);
  return a.Dh == 128 ? launch_kernel("cache_read", cache_read_kernel<128, false>, grid, block, 0, s, a)
                     : launch_kernel("cache_read", cache_read_kernel<64, false>, grid, block, 0, s, a);
}

}  // namespace mapk
