// Attention of new rows over their sequences' cached keys and values.
//
//   out = sum_j p_j v_j / sum_j p_j,  p_j = 2^(c2 <q, k_j> - m),  over the tokens
//   j the row sees; c2 = scale log2(e), m the running maximum (one pass).
//
// Both products are formed transposed on the matrix cores, S^T = K Q^T and
// O^T = V^T P^T, so that a lane holds one query (a column) throughout: the
// maximum and the sums are over its own registers and an exchange or two, the
// statistics and the rescaling are per lane, and the scores become the second
// product's operand in place, its keys taken in the order in which the lane
// holds them.  V passes through LDS row by row as it lies in the pages, and the
// transposing LDS reads (ds_read_b64_tr_b16: 16 lanes give the addresses of 4
// keys' 16 values and get a value's 4 keys each) bring it to that order.
// 4-bit values are widened to bf16 on their way to the registers (keys) or to
// LDS (values), scale and all, which is exact.
//
// The matrix cores take bf16 operands, 2^-8 of a probability's value.  Few rows,
// which the cache's bytes bound, give each as two bf16 numbers (2^-17) and pay
// for the second product with 0 to 5 % (16 single tokens over 2952: 135.6 us, 136.6
// so): their error against 64 bits is that of a float32 softmax, 1.68e-3, all of it
// the output's rounding, where one number gives 2.12e-3.  Prompts, which the matrix
// cores bound, would pay 37 % (2944 rows: 88 us, 120 so) for 1.65e-3 in place of
// 2.06e-3: they give one, and sum what they gave, so that a row's weights add up
// to one and equal values come back as they are (87 us with the sum of the unrounded
// ones).
//
// Output rows are rescaled only when a row's maximum has grown by more than
// 2^6 (the sums carry the same factor, so the result is the same softmax).  m
// starts below every score that counts but finite, so that a row whose scores so
// far are all -inf, or all hidden, has zero probabilities there.
#include <type_traits>

#include "cache_pages.h"

namespace mapk {

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;

constexpr float kLow = -3.0e38f;   // m before the first visible score
constexpr float kRescale = 6.0f;   // log2 of the growth that a row's factor may lag behind
// Sums of finite values may pass float32's range where their mean does not.  A tile
// whose sums come out infinite is run again with its probabilities times 2^-40, for
// up to 2^30 tokens with probabilities up to 2^6; its l is then kept negative, which
// tells the joins.  They form their sums times their `down`, for as many pieces.  All
// of these are powers of two: nothing else about a row changes.
constexpr float kShrink = 0x1p-40f;

// The larger of lanes l and l ^ 32, in both.
__device__ __forceinline__ float max_of_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ s16x4_t tr_read(const void* p) {
  typedef __attribute__((address_space(3))) s16x4_t lds_t;
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (lds_t*)(__attribute__((address_space(3))) void*)const_cast<void*>(p));
}
__device__ __forceinline__ bf16x8_t join(s16x4_t a, s16x4_t b) {
  return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Two bf16 in a word, infinities and NaN cleared.
__device__ __forceinline__ uint32_t word_clean(uint32_t w) {
  if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
  if ((w & 0x7f800000u) == 0x7f800000u) w &= 0xffffu;
  return w;
}
__device__ __forceinline__ bf16x8_t clean8(bf16x8_t v) {
  const uint4 u = __builtin_bit_cast(uint4, v);
  return __builtin_bit_cast(bf16x8_t, make_uint4(word_clean(u.x), word_clean(u.y), word_clean(u.z), word_clean(u.w)));
}

// The exponent of a probability is one multiply-add of a score, which rounds once; m
// was rounded before it.  At scores past 2^26 the two differ by more than the exponents
// of the type: the largest probability is no longer about one.  Such a row shows in
// its l; its tile is run again, with the row's products rounded as m's was.
__device__ __forceinline__ bool far_scores(float m, float l) { return (m > kLow) & !((l >= 0.25f) & (l < INFINITY)); }
__device__ __forceinline__ float exponent_apart(float score, float c2, float m) {
#pragma clang fp contract(off)
  const float x = score * c2;
  return x - m;
}

// s plus eight probabilities, as the second product takes them.
__device__ __forceinline__ float add_weights(bf16x8_t p, float s) {
  const uint4 u = __builtin_bit_cast(uint4, p);
  auto two = [](uint32_t w, float to) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w), __builtin_bit_cast(bf16x2_t, 0x3f803f80u), to, false);
  };
  return s + (two(u.y, two(u.x, 0.0f)) + two(u.w, two(u.z, 0.0f)));
}

// What a piece's sums (m, l) count in a join: mm the largest maximum, shrunk whether
// any piece's l is negative.  (A piece that saw nothing has sums of zero.)
__device__ __forceinline__ float piece_weight(float m, float l, float mm, bool shrunk, float down) {
  return __builtin_amdgcn_exp2f(m - mm) * ((shrunk & (l >= 0.0f)) ? kShrink * down : down);
}

// N values over their sum, as bf16; zeros where nothing was summed.
template <int N> __device__ __forceinline__ void write_row(bf16_t* out, const float* v, float sum) {
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  union { uint2 u[N / 4]; bf16_t e[N]; } w;
#pragma unroll
  for (int k = 0; k < N; ++k) w.e[k] = f32_to_bf16(v[k] * inv);
#pragma unroll
  for (int k = 0; k < N / 4; ++k) reinterpret_cast<uint2*>(out)[k] = w.u[k];
}

// The blocks of KB tokens that rows lo .. hi - 1 (token indices) see any of:
// those of the first tokens, then those from the first row's window to the last row.
struct Blocks {
  int sink, first, count;  // blocks 0 .. sink - 1, then from `first`
  __device__ __forceinline__ int token(int j, int kb) const { return (j < sink ? j : j - sink + first) * kb; }
};
__device__ __forceinline__ Blocks visible_blocks(int lo, int hi, int window, int sinks, int kb) {
  Blocks r;
  const int end = hi > 0 ? (hi + kb - 1) / kb : 0;
  const int from = window > 0 ? max(0, lo - window + 1) / kb : 0;
  r.sink = window > 0 ? min(min(sinks, max(hi, 0)) / kb + (min(sinks, max(hi, 0)) % kb ? 1 : 0), from) : 0;
  r.first = from;
  r.count = r.sink + max(0, end - from);
  return r;
}

// ---------------------------------------------------------------- few rows
// Single tokens and a few rows behind a cache.  The work is one run of blocks: of
// every sequence, key/value head and tile of 16 columns (the (row, query head)
// pairs of that head), the tokens the tile sees.  Each workgroup takes an equal
// stretch of that run, whatever the sequences' lengths; a tile whose blocks lie in
// several stretches leaves its sums for the kernel after it to join.  Within a
// stretch each of the four waves streams every fourth block on its own (no
// barrier until a tile's end).  Bound: the cache's bytes.  A block's keys and values
// come straight to registers (16 bytes a lane: keys as the first product's operand,
// values on their way to LDS), one set of them: the next block's loads leave when
// this one's scores are formed and its values are in LDS, and travel under its softmax
// and second product.  In between a wave has nothing in flight, which the compute
// unit's other seven cover in part: better with bf16 pages, whose scores and LDS writes
// are short (16 single tokens over 2952 of 32 heads, 774 MB: 136.5 us, 5.7 TB/s), than
// with 4-bit ones, which are widened there (32 over 4096 to 32768 of 4 heads, 315 MB: 75 us,
// 4.2 TB/s, and 7.5 for the join).
constexpr int kStepWaves = 4;

template <int DH, bool FP4> struct StepShape {
  static constexpr int KB = FP4 || DH == 64 ? 64 : 32, NT = KB / 16, NM = KB / 32, ND = DH / 16, NS = DH / 32;
  static constexpr int VROW = 2 * DH;                       // bytes of a token's values in LDS
  static constexpr int VPIECE = FP4 ? DH / 2 : 2 * DH;      // and in a page
  static constexpr int NV = KB * VPIECE / 1024;             // 16-byte pieces a lane
  static constexpr int OLD = DH + 4;                        // floats between joined rows
  static constexpr int BYTES = kStepWaves * (KB * VROW > 16 * OLD * 4 ? KB * VROW : 16 * OLD * 4);
};

// Position of 32-byte chunk c of key k's row of V in LDS.  The 32 lanes of half a
// transposing read (8 keys' one chunk, or 4 keys' two) name all 64 banks once, and
// so do 8 lanes that write widened 4-bit values (2 keys' every other chunk).
template <int DH> __device__ __forceinline__ int vchunk(int c, int k) {
  return DH == 128 ? c ^ (((k & 3) << 1) | ((k ^ (k >> 2)) & 1)) : c ^ ((k & 2) | (((k >> 1) ^ (k >> 2)) & 1));
}

// The blocks that column tile ct of a sequence of n rows and len tokens sees.
__device__ __forceinline__ Blocks tile_blocks(const CacheAttnArgs& a, int n, int len, int ct, int kb) {
  const int lo = len - n + 16 * ct / a.G, hi = len - n + min(16 * ct + 15, n * a.G - 1) / a.G + 1;
  return visible_blocks(lo, hi, a.window, a.sinks, kb);
}

// Where each sequence's blocks begin in the run, from the lengths on the device
// (256 threads, one sequence each).
struct StepRun {
  int begin[MAP_CACHE_MAX_BATCH + 1];  // [B]: all blocks
  int wave_sum[4];
  int len[MAP_CACHE_MAX_BATCH], found;
};
__device__ __forceinline__ void lay_out_run(const CacheAttnArgs& a, StepRun& run, int kb) {
  const int t = threadIdx.x, lane = t & 63;
  int v = 0;
  if (t < a.B) {
    const int n = a.off[t + 1] - a.off[t], len = cache_len(a.c, t);
    run.len[t] = len;
    if (n > 0 && n * a.G <= 16)
      v = visible_blocks(len - n, len, a.window, a.sinks, kb).count;
    else if (n > 0 && n <= a.step_rows)
      for (int ct = 0; 16 * ct < n * a.G; ++ct) v += tile_blocks(a, n, len, ct, kb).count;
    v *= a.c.heads;
  }
  int before = v;  // this sequence's and those before it in the wave
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(before, o, 64);
    if (lane >= o) before += u;
  }
  if (lane == 63) run.wave_sum[t >> 6] = before;
  __syncthreads();
  for (int w = 0; w < (t >> 6); ++w) before += run.wave_sum[w];
  if (t < a.B) {
    run.begin[t + 1] = before;
    if (blockIdx.x == 0) {  // (for the kernel that joins)
      a.step_run[2 * t] = before - v;
      a.step_run[2 * t + 1] = run.len[t];
      if (t == a.B - 1) a.step_run[2 * a.B] = before;
    }
  }
  if (t == 0) run.begin[0] = 0;
  __syncthreads();
}
// Equal stretches: the first total % groups are one block longer.
struct Stretches {
  int each, more;
  __device__ __forceinline__ Stretches(int total, int groups) : each(total / groups), more(total % groups) {}
  __device__ __forceinline__ int begin(int w) const { return each * w + min(w, more); }
  __device__ __forceinline__ int of(int x) const {  // the stretch that block x lies in
    return x < more * (each + 1) ? x / (each + 1) : more + (x - more * (each + 1)) / each;
  }
};

template <int DH, bool FP4>  // (2: the launch counts on two workgroups a compute unit)
__global__ __launch_bounds__(64 * kStepWaves, 2) void cache_step_kernel(const CacheAttnArgs a) {
  using X = StepShape<DH, FP4>;
  constexpr int KB = X::KB, NT = X::NT, NM = X::NM, ND = X::ND, NS = X::NS, NV = X::NV;
  __shared__ __attribute__((aligned(1024))) char lds[X::BYTES];
  __shared__ float ms[kStepWaves][16], ls[kStepWaves][16];
  __shared__ StepRun run_of;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lc = lane & 15, g4 = lane >> 4;
  const bool stretch = a.groups > 0;  // (otherwise a workgroup has one tile, and all of it)
  int b, x = 0, x_begin = 0, x_end = 0;
  if (!stretch) {
    b = blockIdx.x / (a.c.heads * a.tiles);
  } else {
    lay_out_run(a, run_of, KB);
    const Stretches all(__builtin_amdgcn_readfirstlane(run_of.begin[a.B]), a.groups);
    x = x_begin = all.begin(blockIdx.x);
    x_end = all.begin(blockIdx.x + 1);
    if (x >= x_end) return;
    if (tid < a.B && run_of.begin[tid] <= x && x < run_of.begin[tid + 1]) run_of.found = tid;
    __syncthreads();
    b = __builtin_amdgcn_readfirstlane(run_of.found);
  }
  for (;;) {
  const int r0 = a.off[b], n = a.off[b + 1] - r0, cols = n * a.G;
  const int len = stretch ? __builtin_amdgcn_readfirstlane(run_of.len[b]) : cache_len(a.c, b);
  int kvh, ct, p0 = 0;
  if (stretch) {
    const int first = __builtin_amdgcn_readfirstlane(run_of.begin[b]), after = __builtin_amdgcn_readfirstlane(run_of.begin[b + 1]);
    const int per_head = (after - first) / a.c.heads;
    kvh = (x - first) / per_head;
    p0 = x - first - kvh * per_head;
    for (ct = 0;; ++ct) {
      const int count = tile_blocks(a, n, len, ct, KB).count;
      if (p0 < count) break;
      p0 -= count;
    }
  } else {
    kvh = blockIdx.x / a.tiles % a.c.heads;
    ct = blockIdx.x % a.tiles;
    if (n > a.step_rows || 16 * ct >= cols) return;
  }
  const int col0 = 16 * ct, base = len - n;  // base: token of the sequence's first new row
  const int i_lo = col0 / a.G, i_hi = min(col0 + 15, cols - 1) / a.G;
  const int lo = base + i_lo, hi = base + i_hi + 1;
  const Blocks blocks = visible_blocks(lo, hi, a.window, a.sinks, KB);
  const int j_end = stretch ? min(blocks.count, p0 + x_end - x) : blocks.count;
  const int j0 = p0 + wave;

  // this lane's query
  const int col = min(col0 + lc, cols - 1), row = col / a.G, head = kvh * a.G + col - row * a.G, me = base + row;
  bf16x8_t qf[NS];
  {
    const bf16_t* q = static_cast<const bf16_t*>(a.q) + (r0 + row) * a.ldq + head * DH;
#pragma unroll
    for (int st = 0; st < NS; ++st)
      qf[st] = *reinterpret_cast<const bf16x8_t*>(q + (FP4 ? (DH / 4) * g4 + 8 * st : 32 * st + 8 * g4));
  }

  // A block on its way: keys as they lie in the pages, values, scale bytes.
  uint4 kr[FP4 ? 1 : NT][FP4 ? 1 : NS], vr[NV];
  uint32_t kw[FP4 ? NT : 1][NS];
  uint32_t ksb[NT], vsb[NV];
  int ent[NT];  // pages of the block's 16-token tiles (-1: none)
  auto load_pages = [&](int t0) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int tok = t0 + 16 * t;
      ent[t] = tok < len ? cache_page(a.c, b, tok) : -1;
    }
  };
  auto tile_row = [&](int t, int t0) {  // (a tile without a page reads the pool's first tokens, masked)
    return ent[t] >= 0 ? cache_row(a.c, ent[t], kvh, t0 + 16 * t) : 0LL;
  };
  auto load_block = [&](int t0) {
    long long rows[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) rows[t] = tile_row(t, t0);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const long long r = rows[t] + lc;
      if constexpr (FP4) {
        const char* p = static_cast<const char*>(a.c.k) + r * (DH / 2) + g4 * (DH / 8);
        if constexpr (DH == 128) {
          const uint4 w = *reinterpret_cast<const uint4*>(p);
          kw[t][0] = w.x;
          kw[t][1] = w.y;
          kw[t][NS - 2] = w.z;
          kw[t][NS - 1] = w.w;
        } else {
          const uint2 w = *reinterpret_cast<const uint2*>(p);
          kw[t][0] = w.x;
          kw[t][1] = w.y;
        }
        ksb[t] = a.c.ks[r * NS + g4 * NS / 4];
      } else {
#pragma unroll
        for (int st = 0; st < NS; ++st)
          kr[t][st] = *reinterpret_cast<const uint4*>(static_cast<const bf16_t*>(a.c.k) + r * DH + 32 * st + 8 * g4);
      }
    }
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      constexpr int PPK = X::VPIECE / 16, KPU = 64 / PPK;  // pieces a key, keys a load
      const int key = u * KPU + lane / PPK, c = lane % PPK;
      long long r = rows[u * KPU / 16];
      if (KPU == 32 && lane >= 32) r = rows[u * KPU / 16 + 1];
      r += key & 15;
      vr[u] = *reinterpret_cast<const uint4*>(static_cast<const char*>(a.c.v) + r * X::VPIECE + 16 * c);
      if constexpr (FP4) vsb[u] = a.c.vs[r * NS + c];
    }
  };

  f32x4_t o[ND];  // O^T: rows 16 d + 4 g4 + (0..3) = values, column lc = the query
  float m, l;
  char* vt = lds + wave * KB * X::VROW;
  const int tr_key = 4 * g4 + (lc >> 2);  // the key and 8 bytes this lane names for a transposing read
  const char* tr_at = vt + tr_key * X::VROW + 8 * (lc & 3);

  // The block's tokens that this lane's row sees, and that any row of the tile sees:
  // from its window on, up to itself, and the first tokens.
  const int from = a.window > 0 ? me - a.window + 1 : 0, from_lo = a.window > 0 ? lo - a.window + 1 : 0;
  auto sees = [&](int cur, int k, uint32_t page) {
    const int tok = cur + k;
    return static_cast<bool>((page != 0u) & (tok <= me) & ((tok >= from) | (tok < a.sinks)));
  };
  bool apart = false;  // this row's scores are far
  auto run = [&](auto careful) {
  m = kLow;
  l = 0.0f;
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  int j = j0, t0 = 0;
  if (j < j_end) {
    t0 = blocks.token(j, KB);
    load_pages(t0);
    load_block(t0);
  }
  while (j < j_end) {
    // what of the block can be seen: all of it by every row, or token by token
    bool pages = true;
    uint32_t held = 0;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      pages = pages && ent[t] >= 0;
      held |= ent[t] >= 0 ? 1u << t : 0u;
    }
    const int cur = t0;
    const bool whole = pages && cur + KB - 1 <= lo && (a.window == 0 || hi - 1 - cur < a.window || cur + KB <= a.sinks);
    // S^T
    f32x4_t sc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      sc[t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int st = 0; st < NS; ++st) {
        bf16x8_t kf;
        if constexpr (FP4) kf = __builtin_bit_cast(bf16x8_t, fp4_eight(kw[t][st], fp4_scale(ksb[t])));
        else kf = __builtin_bit_cast(bf16x8_t, kr[t][st]);
        sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[st], sc[t], 0, 0, 0);
      }
    }
    // V to LDS; a token that no row of the tile sees is zeroed (its values may be anything)
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      constexpr int PPK = X::VPIECE / 16;
      const int key = u * (64 / PPK) + lane / PPK, c = lane % PPK, tok = cur + key;
      if (!whole) {
        if (!(((held >> (key >> 4)) & 1u) & (tok < hi) & ((tok >= from_lo) | (tok < a.sinks)))) {
          vr[u] = make_uint4(0u, 0u, 0u, 0u);
          vsb[u] = 0u;  // (4 bits: zero codes need a scale that is no NaN)
        }
      }
      if constexpr (FP4) {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const uint32_t w = x == 0 ? vr[u].x : x == 1 ? vr[u].y : x == 2 ? vr[u].z : vr[u].w;
          *reinterpret_cast<uint4*>(vt + key * X::VROW + 32 * vchunk<DH>(2 * c + (x >> 1), key) + 16 * (x & 1)) =
              fp4_eight(w, fp4_scale(vsb[u]));
        }
      } else {
        *reinterpret_cast<uint4*>(vt + key * X::VROW + 32 * vchunk<DH>(c >> 1, key) + 16 * (c & 1)) = vr[u];
      }
    }
    // the next block's loads under the rest of this one
    j += kStepWaves;
    if (j < j_end) {
      t0 = blocks.token(j, KB);
      load_pages(t0);
      load_block(t0);
    }
    // the row's maximum and probabilities
    float z[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) z[t][r] = sc[t][r];
    if (!whole) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) z[t][r] = sees(cur, 16 * t + 4 * g4 + r, (held >> t) & 1u) ? z[t][r] : -INFINITY;
    }
    float mx = z[0][0];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, z[t][r]);
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * a.c2;
    const bool grow = mx > m + kRescale;
    if (__any(grow)) {
      const float al = grow ? __builtin_amdgcn_exp2f(m - mx) : 1.0f;  // (first block: 0)
      if (grow) m = mx;
      l *= al;
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] *= al;
    }
    bf16x8_t ph[NM], pl[NM];  // each as two bf16 numbers
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float p = __builtin_amdgcn_exp2f(fmaf(z[t][r], a.c2, -m));
        if constexpr (careful.value) p = kShrink * (apart ? __builtin_amdgcn_exp2f(exponent_apart(z[t][r], a.c2, m)) : p);
        const __bf16 high = static_cast<__bf16>(p);
        l += p;
        ph[t >> 1][4 * (t & 1) + r] = high;
        pl[t >> 1][4 * (t & 1) + r] = static_cast<__bf16>(p - static_cast<float>(high));
      }
    // O^T += V^T P^T
    auto vfrag = [&](int x, int d) {
      const char* at = tr_at + 32 * x * X::VROW + 32 * vchunk<DH>(d, tr_key);
      return join(tr_read(at), tr_read(at + 16 * X::VROW));
    };
    auto weigh = [&](bf16x8_t v, int x, f32x4_t& sum) {
      sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, ph[x], sum, 0, 0, 0);
      sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pl[x], sum, 0, 0, 0);
    };
    if constexpr (careful.value) {
#pragma unroll
      for (int x = 0; x < NM; ++x)
#pragma unroll
        for (int d = 0; d < ND; ++d) weigh(clean8(vfrag(x, d)), x, o[d]);
      for (int k = 0; k < KB; ++k) {
        const bool see = sees(cur, k, (held >> (k >> 4)) & 1u);
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const bf16_t v = *reinterpret_cast<const bf16_t*>(vt + k * X::VROW + 32 * vchunk<DH>(d, k) + 2 * (4 * g4 + r));
            o[d][r] += (see & ((v & 0x7f80) == 0x7f80)) ? bf16_to_f32(v) : 0.0f;
          }
      }
    } else {
#pragma unroll
      for (int x = 0; x < NM; ++x)
#pragma unroll
        for (int d = 0; d < ND; ++d) weigh(vfrag(x, d), x, o[d]);
    }
  }
  };
  // Every value taken as finite; if a sum comes out infinite or NaN, or a row's scores
  // are far (far_scores), once more with smaller probabilities (kShrink), keeping such
  // values from the rows that do not see them (their zero probability would not cancel
  // them): the product runs on the finite values, the others add themselves to the rows
  // that see them.
  run(std::false_type{});
  auto sum_l = [&]() {
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
  };
  sum_l();
  bool shrunk = false;
  {
    apart = far_scores(m, l);
    f32x4_t any = {0.0f, 0.0f, 0.0f, 0.0f};  // NaN once a sum is not finite
#pragma unroll
    for (int d = 0; d < ND; ++d) any += o[d] * 0.0f;
    if (__any(apart | (any[0] + any[1] + any[2] + any[3] != 0.0f))) {
      run(std::true_type{});
      sum_l();
      shrunk = true;
    }
  }

  // join the waves
  if (g4 == 0) {
    ms[wave][lc] = m;
    ls[wave][lc] = shrunk ? -l : l;
  }
  __syncthreads();  // (V is read out)
  float* os = reinterpret_cast<float*>(lds) + wave * 16 * X::OLD;
#pragma unroll
  for (int d = 0; d < ND; ++d) *reinterpret_cast<f32x4_t*>(os + lc * X::OLD + 16 * d + 4 * g4) = o[d];
  __syncthreads();
  constexpr int PER = DH / 16;  // values a thread
  const int c = tid >> 4, d0 = (tid & 15) * PER;
  if (col0 + c < cols) {
    float mm = kLow, sum = 0.0f, v[PER];
    bool any = false;
#pragma unroll
    for (int w = 0; w < kStepWaves; ++w) {
      mm = fmaxf(mm, ms[w][c]);
      any |= ls[w][c] < 0.0f;
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) v[k] = 0.0f;
#pragma unroll
    for (int w = 0; w < kStepWaves; ++w) {
      const float lw = ls[w][c], f = piece_weight(ms[w][c], lw, mm, any, 0x1p-3f);
      if (lw == 0.0f) continue;
      sum = fmaf(f, fabsf(lw), sum);
      const float* src = reinterpret_cast<const float*>(lds) + (w * 16 + c) * X::OLD + d0;
#pragma unroll
      for (int k = 0; k < PER; ++k) v[k] = fmaf(f, src[k], v[k]);
    }
    if (p0 == 0 && j_end == blocks.count) {
      const int rr = (col0 + c) / a.G, hh = kvh * a.G + col0 + c - rr * a.G;
      write_row<PER>(static_cast<bf16_t*>(a.out) + (r0 + rr) * a.ldo + hh * DH + d0, v, sum);
    } else {  // the stretch's first tile, or its last
      const long long at = (2LL * blockIdx.x + (x == x_begin ? 0 : 1)) * 16 + c;
      if (d0 == 0) a.step_ml[at] = make_float2(mm, any ? -sum : sum);
      float4* po = reinterpret_cast<float4*>(a.step_o + at * DH + d0);
#pragma unroll
      for (int k = 0; k < PER / 4; ++k) po[k] = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
    }
  }
  if (!stretch) return;
  x += j_end - p0;
  if (x >= x_end) return;
  __syncthreads();  // (LDS is read out)
  while (x >= __builtin_amdgcn_readfirstlane(run_of.begin[b + 1])) ++b;
  }
}

// The tiles that lie in several stretches: out = sum_s f_s o_s / sum_s f_s l_s over
// their pieces s, f_s = 2^(m_s - max m).  A tile that sees nothing is in none: zeros.
template <int DH, bool FP4>
__global__ __launch_bounds__(256) void cache_step_join_kernel(const CacheAttnArgs a) {
  constexpr int KB = StepShape<DH, FP4>::KB, PER = DH / 16;
  const int b = blockIdx.z, r0 = a.off[b], n = a.off[b + 1] - r0, cols = n * a.G;
  const int kvh = blockIdx.x / a.tiles, ct = blockIdx.x - kvh * a.tiles;
  if (n > a.step_rows || 16 * ct >= cols) return;
  const int len = a.step_run[2 * b + 1];
  int first = a.step_run[2 * b] + kvh * ((a.step_run[2 * b + 2] - a.step_run[2 * b]) / a.c.heads);
  for (int t = 0; t < ct; ++t) first += tile_blocks(a, n, len, t, KB).count;
  const int last = first + tile_blocks(a, n, len, ct, KB).count - 1;
  const Stretches all(a.step_run[2 * a.B], a.groups);
  int w0 = 0, w1 = -1;  // the stretches it lies in
  if (last >= first) {
    w0 = __builtin_amdgcn_readfirstlane(all.of(first));
    w1 = __builtin_amdgcn_readfirstlane(all.of(last));
    if (w0 == w1) return;  // (written whole)
  }
  const int c = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * PER;
  if (16 * ct + c >= cols) return;
  float mm = kLow, sum = 0.0f, v[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) v[k] = 0.0f;
  auto piece = [&](int w) {  // the first tile of its stretch, or the last
    return (2LL * w + (first <= all.begin(w) ? 0 : 1)) * 16 + c;
  };
  float low = 0.0f;  // the least l
#pragma unroll 8
  for (int w = w0; w <= w1; ++w) {
    const float2 ml = a.step_ml[piece(w)];
    mm = fmaxf(mm, ml.x);
    low = fminf(low, ml.y);
  }
#pragma unroll 4
  for (int w = w0; w <= w1; ++w) {
    const float2 ml = a.step_ml[piece(w)];
    const float f = piece_weight(ml.x, ml.y, mm, low < 0.0f, 0x1p-10f);
    const float4* po = reinterpret_cast<const float4*>(a.step_o + piece(w) * DH + d0);
    sum = fmaf(f, fabsf(ml.y), sum);
#pragma unroll
    for (int k = 0; k < PER / 4; ++k) {
      const float4 o = po[k];
      v[4 * k] = fmaf(f, o.x, v[4 * k]);
      v[4 * k + 1] = fmaf(f, o.y, v[4 * k + 1]);
      v[4 * k + 2] = fmaf(f, o.z, v[4 * k + 2]);
      v[4 * k + 3] = fmaf(f, o.w, v[4 * k + 3]);
    }
  }
  const int rr = (16 * ct + c) / a.G, hh = kvh * a.G + 16 * ct + c - rr * a.G;
  write_row<PER>(static_cast<bf16_t*>(a.out) + (r0 + rr) * a.ldo + hh * DH + d0, v, sum);
}

// Joins the parts of the prompts' rows in the same way.
template <int DH>
__global__ __launch_bounds__(256) void cache_prompt_join_kernel(const CacheJoinArgs a) {
  constexpr int LPH = DH / 4;  // lanes a row and head
  const long long item = (long long)blockIdx.x * (256 / LPH) + threadIdx.x / LPH, items = (long long)a.rows * a.Hq;
  if (item >= items) return;
  const int i = static_cast<int>(item / a.Hq), h = static_cast<int>(item - (long long)i * a.Hq), d0 = 4 * (threadIdx.x % LPH);
  int b = 0;  // the row's prompt: the last that starts at or before it
  for (int s = MAP_CACHE_MAX_BATCH / 2; s > 0; s >>= 1)
    if (b + s < a.prompts && a.prompt[b + s].x <= i) b += s;
  const int r = a.prompt[b].y + i - a.prompt[b].x;
  float mm = kLow, low = 0.0f, sum = 0.0f, v[4] = {0.0f, 0.0f, 0.0f, 0.0f};  // low: the least l
  // (a few parts' loads together; past the last, that one's again, unused)
  for (int s0 = 0; s0 < a.parts; s0 += 4) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float2 ml = a.part_ml[(long long)min(s0 + u, a.parts - 1) * items + item];
      mm = fmaxf(mm, ml.x);
      low = fminf(low, ml.y);
    }
  }
  for (int s0 = 0; s0 < a.parts; s0 += 2) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const long long at = (long long)min(s0 + u, a.parts - 1) * items + item;
      const float2 ml = a.part_ml[at];
      const float4 o = *reinterpret_cast<const float4*>(a.part_o + at * DH + d0);
      const bool in = s0 + u < a.parts;
      const float f = piece_weight(ml.x, ml.y, mm, low < 0.0f, 0x1p-7f);
      sum = in ? fmaf(f, fabsf(ml.y), sum) : sum;
      v[0] = in ? fmaf(f, o.x, v[0]) : v[0];  // (no weight of zero: the sums may be infinite)
      v[1] = in ? fmaf(f, o.y, v[1]) : v[1];
      v[2] = in ? fmaf(f, o.z, v[2]) : v[2];
      v[3] = in ? fmaf(f, o.w, v[3]) : v[3];
    }
  }
  write_row<4>(static_cast<bf16_t*>(a.out) + r * a.ldo + h * DH + d0, v, sum);
}

}  // namespace

namespace {

// ---------------------------------------------------------------- prompts
// Workgroup (query block of 128 rows, query head, sequence, part of the tokens);
// wave w owns 32 rows.  64 tokens at a time pass through LDS, two buffers, one
// barrier a block, the next block on its way under this one's products: bf16
// pages by direct loads, 4-bit pages through registers, widened once for all the
// workgroup's rows.  A wave brings the 16 tokens that one table entry names.
// Bound: the clock, which a full card lowers to 1.6 GHz; a block takes a wave 3600
// clocks, 1024 of them matrix instructions, 880 the issue of its loads, and the two
// waves of a SIMD overlap in part.  2944 rows of 32 heads, causal: 89 us (71 GFLOP of
// visible scores, 0.80 PFLOP/s); two prompts of 4700 rows, 28 heads over 4 in 4 bits,
// window 1152: 206 us (0.69 PFLOP/s).  64 rows a wave, one wave a SIMD: 143 for 89 us.
typedef __attribute__((ext_vector_type(16))) float f32x16_t;
constexpr int kKeys = 64;

__device__ const uint4 zero_piece[1] = {};  // what a hidden token's values are loaded from

// Row and column of accumulator register r of lane `lane` in a 32 x 32 matrix-core block.
__device__ __forceinline__ int acc_row(int r, int lane) { return 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3); }

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // M0 is written here and nowhere else in the file
__device__ __forceinline__ void dma16(const void* gsrc, uint32_t m) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(gsrc), "s"(m) : "memory", "m0");
}
// The same with one base address for the wave and an offset a lane.
__device__ __forceinline__ void dma16_from(const void* base, uint32_t off, uint32_t m) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(base), "s"(m) : "memory", "m0");
}
#pragma clang diagnostic pop

// Position of 16-byte chunk c of key k's row of K in LDS.
template <int DH> __device__ __forceinline__ int kchunk(int c, int k) {
  return DH == 128 ? c ^ (k & 15) : c ^ ((k >> 1) & 7);
}

template <int DH, bool FP4>
__global__ __launch_bounds__(256, 2) void cache_prompt_kernel(const CacheAttnArgs a) {
  constexpr int NW = 4, ROW = 2 * DH, BUF = kKeys * ROW, CPR = ROW / 16;  // bytes a token, a buffer; pieces a token
  constexpr int NS = DH / 16, ND = DH / 32;
  __shared__ __attribute__((aligned(1024))) char lds[4 * BUF];  // K, K, V, V
  __shared__ int4 pages[256];
  const int b = blockIdx.z, r0 = a.off[b], n = a.off[b + 1] - r0;
  const int tiles = gridDim.y / a.prompt_splits, part = blockIdx.y % a.prompt_splits;
  const int q0 = (tiles - 1 - static_cast<int>(blockIdx.y) / a.prompt_splits) * 32 * NW;  // the longest first
  if (n <= a.step_rows || q0 >= n) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, lh = lane >> 5, h = blockIdx.x, kvh = h / a.G;
  const int len = cache_len(a.c, b), base = len - n;
  const int lo = base + q0, hi = base + min(q0 + 32 * NW, n);          // the workgroup's tokens
  const int wlo = lo + 32 * wave, whi = min(wlo + 32, base + n);       // this wave's (none if whi <= wlo)
  const int me = wlo + lr, from = a.window > 0 ? me - a.window + 1 : 0;  // this lane's, and its window's first
  const int from_lo = a.window > 0 ? lo - a.window + 1 : 0;
  const Blocks blocks = visible_blocks(lo, hi, a.window, a.sinks, kKeys);
  const int j_begin = static_cast<int>((long long)blocks.count * part / a.prompt_splits);
  const int j_end = static_cast<int>((long long)blocks.count * (part + 1) / a.prompt_splits);

  bf16x8_t qf[NS];  // the query's values 16 st + 8 lh + (0..7)
  {
    const bf16_t* q = static_cast<const bf16_t*>(a.q) + (r0 + min(q0 + 32 * wave + lr, n - 1)) * a.ldq + h * DH + 8 * lh;
#pragma unroll
    for (int st = 0; st < NS; ++st) qf[st] = *reinterpret_cast<const bf16x8_t*>(q + 16 * st);
    // The queries are waited for here: left to their first use, inside the loop, the
    // compiler's waits for them would take in every block on its way to LDS.
#pragma unroll
    for (int st = 0; st < NS; ++st) asm volatile("" : "+v"(qf[st]));
  }
  const uint32_t lds_at = static_cast<uint32_t>(
      reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void*)&lds[0]));
  auto seen = [&](int tok) { return static_cast<bool>((tok < hi) & ((tok >= from_lo) | (tok < a.sinks))); };

  // The pages of up to 256 blocks at a time, four 16-token tiles each (-1: none), in LDS.
  auto fill_pages = [&](int j) {
    const int t0 = j + tid < j_end ? blocks.token(j + tid, kKeys) : len;
    int4 e;
    e.x = t0 < len ? cache_page(a.c, b, t0) : -1;
    e.y = t0 + 16 < len ? cache_page(a.c, b, t0 + 16) : -1;
    e.z = t0 + 32 < len ? cache_page(a.c, b, t0 + 32) : -1;
    e.w = t0 + 48 < len ? cache_page(a.c, b, t0 + 48) : -1;
    pages[tid] = e;
  };
  // Each wave brings 16 of a block's 64 tokens.
  constexpr int PPK = FP4 ? DH / 32 : CPR;          // 16-byte pieces a token in a page
  constexpr int NP = FP4 ? 1 : 16 * PPK / 64;       // pieces a lane, of keys and of values
  constexpr int KPI = FP4 ? 16 : 64 / CPR;          // tokens a piece of all lanes covers
  const int mine = 16 * wave;
  uint4 k_piece, v_piece;  // 4 bits: the pieces on their way
  uint32_t k_byte = 0, v_byte = 0;
  bool vis = false;
  long long row = 0, v_row = 0;  // rows of this wave's first token of the blocks whose keys, values come next,
  bool has = false, v_has = false;  // and whether it has a page
  uint32_t have = 0;  // four bits for each of the last blocks found, the latest lowest: which 16-token tiles have a page
  auto find = [&](int j) {  // a tile without a page reads the pool's first tokens, masked
    const int4 e = pages[(j - j_begin) & 255];
    const int own = wave == 0 ? e.x : wave == 1 ? e.y : wave == 2 ? e.z : e.w;
    const int page = __builtin_amdgcn_readfirstlane(j < j_end ? own : -1);
    have = (have << 4) |
           __builtin_amdgcn_readfirstlane((e.x >= 0 ? 1 : 0) | (e.y >= 0 ? 2 : 0) | (e.z >= 0 ? 4 : 0) | (e.w >= 0 ? 8 : 0));
    v_row = row;
    v_has = has;
    has = page >= 0;
    row = has ? cache_row(a.c, page, kvh, blocks.token(j, kKeys) + mine) : 0LL;
  };
  const int p_key = FP4 ? lane / PPK % 16 : lane / CPR, p_at = FP4 ? lane % PPK : lane % CPR;
  auto load_k = [&](int j) {
    if constexpr (FP4) {
      const long long r = row + p_key;
      k_piece = *reinterpret_cast<const uint4*>(static_cast<const char*>(a.c.k) + r * (DH / 2) + 16 * p_at);
      k_byte = a.c.ks[r * PPK + p_at];
    } else {
#pragma unroll
      for (int u = 0; u < NP; ++u)
        dma16_from(static_cast<const char*>(a.c.k) + row * ROW,
                   (KPI * u + p_key) * ROW + 16 * kchunk<DH>(p_at, KPI * u + p_key),
                   lds_at + static_cast<uint32_t>(j & 1) * BUF + 1024u * (wave * NP + u));
    }
  };
  auto load_v = [&](int j) {
    const int t0 = blocks.token(j, kKeys) + mine;
    if constexpr (FP4) {
      const long long r = v_row + p_key;
      v_piece = *reinterpret_cast<const uint4*>(static_cast<const char*>(a.c.v) + r * (DH / 2) + 16 * p_at);
      v_byte = a.c.vs[r * PPK + p_at];
      vis = v_has & seen(t0 + p_key);
    } else {
      const char* base = static_cast<const char*>(a.c.v) + v_row * ROW;
      const uint32_t to = lds_at + static_cast<uint32_t>(2 + (j & 1)) * BUF + 1024u * (wave * NP);
      if (v_has & (t0 + 15 < hi) & ((t0 >= from_lo) | (t0 + 15 < a.sinks))) {
#pragma unroll
        for (int u = 0; u < NP; ++u)
          dma16_from(base, (KPI * u + p_key) * ROW + 32 * vchunk<DH>(p_at >> 1, KPI * u + p_key) + 16 * (p_at & 1), to + 1024u * u);
      } else {  // a token that no row of the workgroup sees: zeros, whatever its values are
#pragma unroll
        for (int u = 0; u < NP; ++u) {
          const int key = KPI * u + p_key;
          const char* v = base + key * ROW + 32 * vchunk<DH>(p_at >> 1, key) + 16 * (p_at & 1);
          dma16((v_has & seen(t0 + key)) ? v : reinterpret_cast<const char*>(zero_piece), to + 1024u * u);
        }
      }
    }
  };
  // 4 bits: the piece to LDS, as bf16 (head_dim 64: 32 lanes hold the 16 tokens, the others repeat them)
  auto store_k = [&](int j) {
    const uint32_t w[4] = {k_piece.x, k_piece.y, k_piece.z, k_piece.w};
    char* at = lds + (j & 1) * BUF + (mine + p_key) * ROW;
    if (PPK == 4 || lane < 16 * PPK)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        *reinterpret_cast<uint4*>(at + 16 * kchunk<DH>(4 * p_at + x, mine + p_key)) = fp4_eight(w[x], fp4_scale(k_byte));
  };
  auto store_v = [&](int j) {
    const uint32_t w[4] = {v_piece.x, v_piece.y, v_piece.z, v_piece.w};
    char* at = lds + (2 + (j & 1)) * BUF + (mine + p_key) * ROW;
    if (PPK == 4 || lane < 16 * PPK)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        *reinterpret_cast<uint4*>(at + 32 * vchunk<DH>(2 * p_at + (x >> 1), mine + p_key) + 16 * (x & 1)) =
            vis ? fp4_eight(w[x], fp4_scale(v_byte)) : make_uint4(0u, 0u, 0u, 0u);
  };
  // Every wave's loads are here, and its reads of the block before done.
  auto meet = [&]() {
    if constexpr (FP4) __syncthreads();
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory");
  };

  // The step behind the last half of a block (32 tokens, counted from the first
  // block of the run) that holds something for this wave: there is none after it.
  const int last = whi > max(wlo, 0) ? min(2 * j_end, 2 * (blocks.sink - blocks.first) + (whi - 1) / 32 + 1) : -2;

  f32x16_t o[ND];  // O^T: rows 32 d + acc_row = values, column lr = the query
  float m, l;
  const float c2 = a.c2;
  bool apart = false;  // this row's scores are far
  const int tr_key = 4 * lh + ((lane & 15) >> 2);
  auto token_of = [&](int i) { return blocks.token(i >> 1, kKeys) + 32 * (i & 1); };
  // S^T of half i: rows = keys acc_row, column = the query
  auto scores = [&](int i, f32x16_t& sc) {
    const char* K = lds + ((i >> 1) & 1) * BUF + 32 * (i & 1) * ROW;
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[r] = 0.0f;
#pragma unroll
    for (int st = 0; st < NS; ++st)
      sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          *reinterpret_cast<const bf16x8_t*>(K + lr * ROW + 16 * kchunk<DH>(2 * st + lh, lr)), qf[st], sc, 0, 0, 0);
  };
  auto visible = [&](int cur, uint32_t two, int k) {
    const int tok = cur + k;
    return static_cast<bool>(((two >> (k >> 4)) & 1u) & (tok <= me) & ((tok >= from) | (tok < a.sinks)));
  };
  // Step i, between the scores of half i (formed in the step before) and its sums
  // (formed in the next): half i's maximum; then, independent of each other, half
  // i + 1's scores, half i's probabilities and the sums of half i - 1; then the
  // rescaling, if the maximum has grown.  `two`, `two_before`: which 16-token tiles
  // of half i, i - 1 have a page.
  auto step = [&](int i, uint32_t two, uint32_t two_before, f32x16_t& sc, f32x16_t& next, bf16x8_t (&p)[2],
                  const bf16x8_t (&before)[2], auto careful) {
    {
      const int cur = token_of(i);
      const bool whole = two == 3u && i < 2 * j_end && cur + 31 <= wlo &&
                         (a.window == 0 || whi - 1 - cur < a.window || cur + 32 <= a.sinks);
      if (!whole) {
        const uint32_t any = i < 2 * j_end ? two : 0u;  // (behind the last half: nothing)
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] = visible(cur, any, acc_row(r, lane)) ? sc[r] : -INFINITY;
      }
    }
    // (The half before's, up here, where they are long there: 2944 rows 87.1 us and two
    // video prompts 202.3; summed right behind their exponentials, 88.3 and 204.9; the
    // unrounded ones, 86.2 and 200.2, on that card.)
    l = add_weights(before[1], add_weights(before[0], l));
    float mx = sc[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, sc[r]);
    mx = max_of_halves(mx) * c2;
    const bool grow = mx > m + kRescale;
    const float m_before = m;
    if (grow) m = mx;

    scores(i + 1, next);  // (behind the last half: unused)
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        float e = __builtin_amdgcn_exp2f(fmaf(sc[8 * st + k], c2, -m));
        if constexpr (careful.value) e = kShrink * (apart ? __builtin_amdgcn_exp2f(exponent_apart(sc[8 * st + k], c2, m)) : e);
        p[st][k] = static_cast<__bf16>(e);
      }
    const char* V = lds + (2 + (((i - 1) >> 1) & 1)) * BUF + 32 * ((i - 1) & 1) * ROW;
    auto vfrag = [&](int st, int d) {  // keys 16 st + 4 lh + (0..3) and + 8, value 32 d + lr
      const char* at = V + (16 * st + tr_key) * ROW + 8 * (lane & 3);
      const int c = 2 * d + ((lane >> 4) & 1);
      return join(tr_read(at + 32 * vchunk<DH>(c, tr_key)), tr_read(at + 8 * ROW + 32 * vchunk<DH>(c, tr_key + 8)));
    };
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        bf16x8_t v = vfrag(st, d);
        if constexpr (careful.value) v = clean8(v);
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, before[st], o[d], 0, 0, 0);
      }
    if constexpr (careful.value) {
      const int cur = token_of(i - 1);
      for (int k = 0; k < 32; ++k) {
        const bool see = (i > 2 * j_begin) & visible(cur, two_before, k);
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int dim = 32 * d + acc_row(r, lane);
            const bf16_t v = *reinterpret_cast<const bf16_t*>(V + k * ROW + 32 * vchunk<DH>(dim >> 4, k) + 2 * (dim & 15));
            o[d][r] += (see & ((v & 0x7f80) == 0x7f80)) ? bf16_to_f32(v) : 0.0f;
          }
      }
    }
    // (the exponentials stay up here, beside the products, and do not sink below the branch)
    asm volatile("" : "+v"(p[0]), "+v"(p[1]));
    if (__any(grow)) {
      const float al = grow ? __builtin_amdgcn_exp2f(m_before - m) : 1.0f;  // (first block: 0)
      l *= al;
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] *= al;
    }
  };
  // Keys of block j are read in steps 2 j - 1 and 2 j, its values in steps 2 j + 1
  // and 2 j + 2: so one meeting a block, before an odd step, that brings the keys of
  // the block after next and the values of the next.
  // A first run takes every value as finite; if a sum comes out infinite or NaN, or a
  // row's scores are far (far_scores), a second one has smaller probabilities (kShrink)
  // and keeps such values from the rows that do not see them (their zero probability
  // would not cancel them): the product runs on the finite values, and the others add
  // themselves to the rows that see them.
  auto run = [&](auto careful) {
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] = 0.0f;
    m = kLow;
    l = 0.0f;
    // (before the first half: no scores, no probabilities)
    f32x16_t even, odd;
    bf16x8_t p_even[2], p_odd[2];
#pragma unroll
    for (int r = 0; r < 16; ++r) odd[r] = -INFINITY;
#pragma unroll
    for (int st = 0; st < 2; ++st) p_even[st] = __builtin_bit_cast(bf16x8_t, make_uint4(0u, 0u, 0u, 0u));
    if (j_begin < j_end) {
      fill_pages(j_begin);
      // (values of the block before the first: zeros, which that zero probability meets)
#pragma unroll
      for (int u = 0; u < BUF / 4096; ++u)
        *reinterpret_cast<uint4*>(lds + (2 + ((j_begin - 1) & 1)) * BUF + 16 * (tid + 256 * u)) = make_uint4(0u, 0u, 0u, 0u);
      __syncthreads();
      find(j_begin);
      load_k(j_begin);
      if constexpr (FP4) store_k(j_begin);
      for (int j = j_begin - 1; j < j_end; ++j) {
        meet();
        if (((j + 2 - j_begin) & 255) == 0) {
          fill_pages(j + 2);
          __syncthreads();
        }
        find(j + 2);
        load_k(j + 2);  // (past the last block: the pool's first tokens, unused)
        load_v(j + 1);
        // have: block j + 2's tiles in bits 0-3, j + 1's in 4-7, j's in 8-11
        if (2 * j + 1 <= last) {
          // (ahead of the other workgroup's wave while that brings its blocks: 2944 rows
          // 89.2 -> 86.7 us; with 4-bit pages, whose widening is vector work, 206 -> 210)
          if constexpr (!FP4) __builtin_amdgcn_s_setprio(1);
          step(2 * j + 1, (have >> 10) & 3u, (have >> 8) & 3u, odd, even, p_odd, p_even, careful);
          step(2 * j + 2, (have >> 4) & 3u, (have >> 10) & 3u, even, odd, p_even, p_odd, careful);
          if constexpr (!FP4) __builtin_amdgcn_s_setprio(0);
        }
        if constexpr (FP4) {
          store_k(j + 2);
          store_v(j + 1);
        }
      }
    }
    float any = 0.0f;  // NaN once a sum is not finite
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) any = fmaf(o[d][r], 0.0f, any);
    apart = far_scores(m, l + __shfl_xor(l, 32, 64));
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): nothing on its way to LDS
    return __syncthreads_or((apart | (any != 0.0f)) & (q0 + 32 * wave + lr < n));  // (and K and V are read out)
  };
  const bool shrunk = run(std::false_type{});
  if (shrunk) run(std::true_type{});
  if (whi <= wlo) return;
  l += __shfl_xor(l, 32, 64);
  const int i = q0 + 32 * wave + lr;  // this lane's row
  if (a.prompt_splits > 1) {
    int before = 0, all = 0;  // rows of the prompts before this one, and of all
    for (int c = lane; c < a.B; c += 64) {
      const int rows = a.off[c + 1] - a.off[c], of = rows > a.step_rows ? rows : 0;
      before += c < b ? of : 0;
      all += of;
    }
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) {
      before += __shfl_xor(before, x, 64);
      all += __shfl_xor(all, x, 64);
    }
    if (i >= n) return;
    const long long at = ((long long)part * all + before + i) * a.Hq + h;
    if (lh == 0) a.part_ml[at] = make_float2(m, shrunk ? -l : l);
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<float4*>(a.part_o + at * DH + 32 * d + 8 * g + 4 * lh) =
            make_float4(o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]);
    return;
  }
  // each wave's output rows through LDS, 8 values more apart than they are long
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  bf16_t* ot = reinterpret_cast<bf16_t*>(lds) + wave * 32 * (DH + 8);
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      ushort4 w;
      w.x = f32_to_bf16(o[d][4 * g] * inv);
      w.y = f32_to_bf16(o[d][4 * g + 1] * inv);
      w.z = f32_to_bf16(o[d][4 * g + 2] * inv);
      w.w = f32_to_bf16(o[d][4 * g + 3] * inv);
      *reinterpret_cast<ushort4*>(ot + lr * (DH + 8) + 32 * d + 8 * g + 4 * lh) = w;
    }
  constexpr int LPR = DH / 8, RPI = 64 / LPR;  // lanes a row, rows at a time
  bf16_t* out = static_cast<bf16_t*>(a.out) + (long long)(r0 + q0 + 32 * wave) * a.ldo + h * DH;
#pragma unroll
  for (int u = 0; u < 32 / RPI; ++u) {  // (this wave's own rows: no barrier)
    const int r = RPI * u + lane / LPR, c = 8 * (lane % LPR);
    if (q0 + 32 * wave + r < n)
      *reinterpret_cast<uint4*>(out + (long long)r * a.ldo + c) = *reinterpret_cast<const uint4*>(ot + r * (DH + 8) + c);
  }
}

// Sequences of up to so many new rows run on the kernel for few rows: its tiles
// of 16 (row, head) pairs read the cache once each, n G / 16 times a key/value
// head, the other kernel once for each of the G heads, with a quarter of its waves
// at work up to 32 rows.  Behind 8000 tokens, few rows' kernel / prompts' (us):
//   rows                       2         8         16         32         64
//   32 heads over 32        35 / 33   37 / 34   38 / 35    45 / 35    67 / 39
//   28 heads over 4         27 / 31   33 / 31   37 / 32    49 / 32    68 / 37
//   8 sequences of these          (4: 45 / 137)  143 / 138  206 / 139  343 / 147
// and behind 300 tokens, 32 over 32: 10 / 13 at 4 and at 16 rows, 10 / 16 at 32.  The
// two cross between 8 and 24 rows in all but that short one.
constexpr int kStepRows = 16;

}  // namespace

// The few rows' workgroups: two a compute unit hold the card, each with an equal
// stretch; fewer where the longest table gives a stretch under eight blocks (4, 8 and 16:
// 16.5, 16.5, 17.6 us for a token of 28 heads over 4 behind 600, 24.9, 25.1, 24.1 for 8
// behind 3000) or a tile over 64 pieces (32, 64 and 128: 36, 41, 52 us behind 30000, 92,
// 74, 94 behind 120000).  Without stretches (0: a workgroup a tile, and no second launch)
//   where no row sees over 512 tokens (one token of 32 heads behind 250, 500, 700, 1000
//   and 2000: 10.3, 11.4, 14.2, 18.5, 33.2 us in tiles, 13.0, 13.6, 17.1, 14.6, 19.2 in
//   stretches);
//   where there is a tile for each place on the card.  That is the better one for
//   lengths that are alike and for many tiles (16 single tokens over 3000 of 32 heads
//   139 us in tiles, 143 in stretches; 128 over 100 to 2000: 368 and 428; 256 over 3000 of 8
//   heads of 64 in 4 bits: 118 and 142), and the worse one just past a full round (17 over
//   2000 of 32 heads: 125 and 109) and for one sequence far longer than the rest, whose
//   tiles then run alone (64 sequences of 8 heads, 63 of 200 tokens and one of 32768: 590
//   and 68).  The lengths are on the device, so the host takes the common case;
//   and where the run might pass 2^30 blocks, which are counted in an int (a window may
//   bring it back, so the workspace has the room).
// Prompts: two workgroups a compute unit, by splitting the tokens where there are
// fewer tiles, 512 tokens a part at least (256, 512 and 1024: 24.6, 23.5, 36.7 us for 40
// rows of 32 heads behind 2500, 30.3, 28.7, 41.3 for 500 of 8 behind 2000; 18.7, 25.8,
// 25.8 for 40 of 8 behind 800).
// tokens: the most that a row can see.
CacheAttnPlan cache_attention_plan(const int* off, int B, int Hq, int Hkv, int Dh, bool fp4, long long tokens, int cus) {
  CacheAttnPlan p{};
  const int G = Hq / Hkv;
  long long step_tiles = 0, prompt_tiles = 0;
  for (int b = 0; b < B; ++b) {
    const int n = off[b + 1] - off[b];
    if (n == 0) continue;
    if (n <= kStepRows) {
      p.step_most = max(p.step_most, n);
      step_tiles += (long long)((n * G + 15) / 16) * Hkv;
    } else {
      p.prompt_most = max(p.prompt_most, n);
      p.prompt_rows += n;
      prompt_tiles += (long long)((n + 127) / 128) * Hq;
    }
  }
  p.tiles = max(1, (p.step_most * G + 15) / 16);
  const long long places = 2LL * cus;
  if (step_tiles > 0 && tokens > 512 && step_tiles < places) {
    const long long blocks = (tokens + 31) / (fp4 || Dh == 64 ? 64 : 32);
    p.groups = static_cast<int>(max(1LL, min(min(places, 64 * step_tiles), step_tiles * blocks / 8)));
    p.run_fits = step_tiles * blocks < 1LL << 30;
  }
  p.prompt_splits = 1;
  if (prompt_tiles > 0) p.prompt_splits = static_cast<int>(max(1LL, min(min(places / prompt_tiles, tokens / 512), 64LL)));
  return p;
}

hipError_t launch_cache_attention(CacheAttnArgs& a, const CacheAttnPlan& p, hipStream_t s) {
  const int groups = p.run_fits ? p.groups : 0;
  a.tiles = p.tiles;
  a.step_rows = kStepRows;
  a.groups = groups;
  a.prompt_splits = p.prompt_splits;
  hipError_t e = hipSuccess;
  const dim3 block(256), tiles(a.c.heads * p.tiles, 1, a.B);  // the join's; the kernel itself counts them in one row
  if (p.step_most > 0) {
    const dim3 grid(groups > 0 ? groups : a.B * a.c.heads * p.tiles);
    if (a.fp4)
      e = a.Dh == 128 ? launch_kernel("cache_step", cache_step_kernel<128, true>, grid, block, 0, s, a)
                      : launch_kernel("cache_step", cache_step_kernel<64, true>, grid, block, 0, s, a);
    else
      e = a.Dh == 128 ? launch_kernel("cache_step", cache_step_kernel<128, false>, grid, block, 0, s, a)
                      : launch_kernel("cache_step", cache_step_kernel<64, false>, grid, block, 0, s, a);
  }
  if (e == hipSuccess && groups > 0) {
    if (a.fp4)
      e = a.Dh == 128 ? launch_kernel("cache_step_join", cache_step_join_kernel<128, true>, tiles, block, 0, s, a)
                      : launch_kernel("cache_step_join", cache_step_join_kernel<64, true>, tiles, block, 0, s, a);
    else
      e = a.Dh == 128 ? launch_kernel("cache_step_join", cache_step_join_kernel<128, false>, tiles, block, 0, s, a)
                      : launch_kernel("cache_step_join", cache_step_join_kernel<64, false>, tiles, block, 0, s, a);
  }
  if (e == hipSuccess && p.prompt_most > 0) {
    const dim3 grid(a.Hq, (p.prompt_most + 127) / 128 * p.prompt_splits, a.B);
    if (a.fp4)
      e = a.Dh == 128 ? launch_kernel("cache_prompt", cache_prompt_kernel<128, true>, grid, block, 0, s, a)
                      : launch_kernel("cache_prompt", cache_prompt_kernel<64, true>, grid, block, 0, s, a);
    else
      e = a.Dh == 128 ? launch_kernel("cache_prompt", cache_prompt_kernel<128, false>, grid, block, 0, s, a)
                      : launch_kernel("cache_prompt", cache_prompt_kernel<64, false>, grid, block, 0, s, a);
    if (e == hipSuccess && p.prompt_splits > 1) {
      CacheJoinArgs j{a.out, a.ldo, a.part_o, a.part_ml, a.Hq, p.prompt_splits, 0, 0, {}};
      for (int b = 0; b < a.B; ++b) {
        const int n = a.off[b + 1] - a.off[b];
        if (n <= kStepRows) continue;
        j.prompt[j.prompts++] = make_int2(j.rows, a.off[b]);
        j.rows += n;
      }
      const long long items = (long long)j.rows * a.Hq, per = 256 / (a.Dh / 4);
      const dim3 joins(static_cast<unsigned>((items + per - 1) / per));
      e = a.Dh == 128 ? launch_kernel("cache_prompt_join", cache_prompt_join_kernel<128>, joins, block, 0, s, j)
                      : launch_kernel("cache_prompt_join", cache_prompt_join_kernel<64>, joins, block, 0, s, j);
    }
  }
  return e;
}

}  // namespace mapk
