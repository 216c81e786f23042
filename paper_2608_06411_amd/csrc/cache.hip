// Rows of keys and values to the pages of a cache and back.
//
// Both directions move 16 bytes (eight bf16 values) a lane, head_dim / 8 lanes a
// (row, head) pair.  A workgroup takes up to 16 consecutive new rows of one
// sequence, each lane one row and every so many heads of it: the rows of a head lie
// next to each other in a page, so what a workgroup writes (reads) there at a time
// is contiguous, and a cache line of 4-bit codes or of scale bytes, which holds
// several tokens, is written by one compute unit and not by several dies' L2 caches
// in turn; and a lane looks its row's page up once.  Bound: the bytes, 2 rows
// (keys, values) read and written; the next pair is loaded before one is stored.
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

// The row (of its tile) and the heads of a lane's pair: rows = the tile's rows
// rounded up to a power of two side by side, the other lanes further heads.
struct Pair {
  int row, head, step;  // head, head + step, ...
  __device__ __forceinline__ Pair(int nt, int pairs, int lanes, int part, int parts) {
    const int shift = nt > 8 ? 4 : nt > 4 ? 3 : nt > 2 ? 2 : nt > 1 ? 1 : 0, g = threadIdx.x / lanes;
    row = g & ((1 << shift) - 1);
    head = (g >> shift) + part * (pairs >> shift);
    step = parts * (pairs >> shift);
  }
};

template <int DH, bool FP4>
__global__ __launch_bounds__(NT) void cache_append_kernel(const CacheRowsArgs a) {
  constexpr int LPH = DH / 8, PAIRS = NT / LPH;  // lanes a (head, row) pair, pairs at a time
  const int b = blockIdx.z, r0 = a.off[b], n = a.off[b + 1] - r0;
  const int t0 = blockIdx.x * kTile, nt = min(kTile, n - t0);
  if (nt <= 0) return;
  const Pair p(nt, PAIRS, LPH, blockIdx.y, a.parts);
  const int l = threadIdx.x % LPH, i = t0 + p.row, j = cache_len(a.c, b) - n + i;
  // (a pair's lanes are all here or all away: the exchange below stays within them)
  const int page = p.row < nt && j >= 0 ? cache_page(a.c, b, j) : -1;
  if (page < 0) return;
  const bf16_t* src_k = static_cast<const bf16_t*>(a.k) + (r0 + i) * a.ldk + 8 * l;
  const bf16_t* src_v = static_cast<const bf16_t*>(a.v) + (r0 + i) * a.ldv + 8 * l;
  Eight k, v;
  if (p.head < a.c.heads) {
    k.u = *reinterpret_cast<const uint4*>(src_k + p.head * DH);
    v.u = *reinterpret_cast<const uint4*>(src_v + p.head * DH);
  }
  for (int h = p.head; h < a.c.heads; h += p.step) {
    const Eight kc = k, vc = v;
    if (h + p.step < a.c.heads) {
      k.u = *reinterpret_cast<const uint4*>(src_k + (h + p.step) * DH);
      v.u = *reinterpret_cast<const uint4*>(src_v + (h + p.step) * DH);
    }
    const long long row = cache_row(a.c, page, h, j);
    if constexpr (!FP4) {
      *reinterpret_cast<uint4*>(static_cast<bf16_t*>(a.c.k) + row * DH + 8 * l) = kc.u;
      *reinterpret_cast<uint4*>(static_cast<bf16_t*>(a.c.v) + row * DH + 8 * l) = vc.u;
    } else {
      uint32_t mk = amax_bits(kc), mv = amax_bits(vc);
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) {
        mk = max(mk, static_cast<uint32_t>(__shfl_xor(static_cast<int>(mk), o, 64)));
        mv = max(mv, static_cast<uint32_t>(__shfl_xor(static_cast<int>(mv), o, 64)));
      }
      const uint32_t bk = fp4_byte(mk), bv = fp4_byte(mv);
      static_cast<uint32_t*>(a.c.k)[row * LPH + l] = fp4_codes(kc, bk);
      static_cast<uint32_t*>(a.c.v)[row * LPH + l] = fp4_codes(vc, bv);
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
  const Pair p(nt, PAIRS, LPH, blockIdx.y, a.parts);
  if (p.row >= nt) return;
  const int l = threadIdx.x % LPH, i = t0 + p.row, j = a.slots ? a.slots[r0 + i] : i;
  const int page = j >= 0 && j < cache_len(a.c, b) ? cache_page(a.c, b, j) : -1;
  bf16_t* dst_k = static_cast<bf16_t*>(a.k) + (r0 + i) * a.ldk + 8 * l;
  bf16_t* dst_v = static_cast<bf16_t*>(a.v) + (r0 + i) * a.ldv + 8 * l;
  Eight k, v;
  uint32_t kw = 0, vw = 0, kb = 0, vb = 0;
  k.u = v.u = make_uint4(0u, 0u, 0u, 0u);
  auto load = [&](int h) {  // (no page: zeros stay)
    if (page < 0 || h >= a.c.heads) return;
    const long long row = cache_row(a.c, page, h, j);
    if constexpr (!FP4) {
      k.u = *reinterpret_cast<const uint4*>(static_cast<const bf16_t*>(a.c.k) + row * DH + 8 * l);
      v.u = *reinterpret_cast<const uint4*>(static_cast<const bf16_t*>(a.c.v) + row * DH + 8 * l);
    } else {
      kw = static_cast<const uint32_t*>(a.c.k)[row * LPH + l];
      vw = static_cast<const uint32_t*>(a.c.v)[row * LPH + l];
      kb = a.c.ks[row * (DH / 32) + l / 4];
      vb = a.c.vs[row * (DH / 32) + l / 4];
    }
  };
  load(p.head);
  for (int h = p.head; h < a.c.heads; h += p.step) {
    Eight kc = k, vc = v;
    if constexpr (FP4) {
      kc.u = fp4_eight(kw, fp4_scale(kb));
      vc.u = fp4_eight(vw, fp4_scale(vb));
    }
    load(h + p.step);
    *reinterpret_cast<uint4*>(dst_k + h * DH) = kc.u;
    *reinterpret_cast<uint4*>(dst_v + h * DH) = vc.u;
  }
}

// Tiles of the longest sequence, and workgroups a tile, so that there are about
// `want` of them (one round of heads each at least).  Writing gains by many short
// ones, reading by few long ones (11776 rows of 32 heads in bf16: append 102 us with
// 512 wanted, 82 with 4096, 78 with 8192; read 76, 82, 82).
dim3 rows_grid(CacheRowsArgs& a, long long want) {
  long long most = 0, tiles = 0;
  for (int b = 0; b < a.B; ++b) {
    const int n = a.off[b + 1] - a.off[b];
    most = max(most, (long long)n);
    tiles += (n + kTile - 1) / kTile;
  }
  const int side = most > 8 ? 16 : most > 4 ? 8 : most > 2 ? 4 : most > 1 ? 2 : 1;  // rows side by side
  const int heads = NT / (a.Dh / 8) / side, rounds = (a.c.heads + heads - 1) / heads;
  a.parts = static_cast<int>(max(1LL, min((long long)rounds, want / max(tiles, 1LL))));
  return dim3(static_cast<unsigned>((most + kTile - 1) / kTile), a.parts, a.B);
}

}  // namespace

hipError_t launch_cache_append(CacheRowsArgs& a, hipStream_t s) {
  const dim3 grid = rows_grid(a, 8192), block(NT);
  if (a.fp4)
    return a.Dh == 128 ? launch_kernel("cache_append", cache_append_kernel<128, true>, grid, block, 0, s, a)
                       : launch_kernel("cache_append", cache_append_kernel<64, true>, grid, block, 0, s, a);
  return a.Dh == 128 ? launch_kernel("cache_append", cache_append_kernel<128, false>, grid, block, 0, s, a)
                     : launch_kernel("cache_append", cache_append_kernel<64, false>, grid, block, 0, s, a);
}

hipError_t launch_cache_read(CacheRowsArgs& a, hipStream_t s) {
  const dim3 grid = rows_grid(a, 512), block(NT);
  if (a.fp4)
    return a.Dh == 128 ? launch_kernel("cache_read", cache_read_kernel<128, true>, grid, block, 0, s, a)
                       : launch_kernel("cache_read", cache_read_kernel<64, true>, grid, block, 0, s, a);
  return a.Dh == 128 ? launch_kernel("cache_read", cache_read_kernel<128, false>, grid, block, 0, s, a)
                     : launch_kernel("cache_read", cache_read_kernel<64, false>, grid, block, 0, s, a);
}

}  // namespace mapk
