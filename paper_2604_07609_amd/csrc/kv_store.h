// Queries, keys and values of an iteration on their way from the projections to the attention: queries and keys normed per head
// (root mean square over the head's dimensions, times a gain), rotated by their positions (pairs i, i + hd/2), the queries
// scaled and written as halves, keys and values stored into the paged cache, in one pass. A cache holds 16 tokens per block:
//
//   16 bits   K [block][kv head][16 tokens][hd], behind it V [block][kv head][hd][16 tokens], halves (the engine's layout)
//   4 bits    a record of 17 hd bytes per (block, kv head): K codes [16 tokens][hd/2], V codes [token / 4][16][token % 4][hd/32] where
//             byte (j, m) holds dimensions 2 (j hd/32 + m) and the next, K scales [hd/32][16 tokens], V scales [hd/32][16 tokens].
//             A code is an e2m1 number (0 .5 1 1.5 2 3 4 6 and their negatives), the lower half of a byte the lower dimension; a
//             scale byte is the exponent + 127 of the power of two that 32 neighbouring dimensions of a token share, 255: not a
//             number. The layout is what a lane of the attention reads with one load: 16 bytes of a key (one scale), and
//             of a value the same 8 dimensions of 4 tokens.
//
// Bound by bytes: each projection is read once, each output written once. 8191 tokens of 32 query and 8 key heads of 128, 206 MB, take
// 43 us (4.8 TB/s, what a plain copy of as much reaches), into 4 bits 43 us for 176 MB. It took 67 us with two rows a lane and 8-byte
// loads, 56 with 17 and not 34 KB of LDS a workgroup, 51 with one row a lane (64 registers: 8 waves a SIMD) and 16-byte loads, 47 with
// non-temporal loads, and 43 with keys apart from queries. Few tokens are bound by their chain (place and position, table, store) and
// the launch: 3 us. What is between the bytes is 32-bit arithmetic, with one exception: keys that go into 4 bits are normed and
// rotated in 64 bits, because a sum in another order would move the few values next to a border between two codes by half their
// size. (Values are not computed on: their codes are exact either way.)
#pragma once
#include "blink_device.h"

#define KV_E_MIN (-23)      // exponents of 4-bit scales: with these every value is a half, exactly
#define KV_E_MAX 13

struct StoreArgs {
  const void *q, *k, *v;          // [token][head][hd], stride between tokens in elements
  u64 qs, ks, vs;
  const float *qg, *kg;           // gains of the norms [hd] (null: not normed)
  const i32 *pos, *slot;          // position of every token and its place in the cache (block * 16 + offset; outside the cache: not stored)
  const float2* tab;              // [rows][hd/2] (cos, sin)
  u32 rows;
  f16_t* qo;                      // queries out
  u64 qos;
  void* cache;
  u32 n_blocks, nq, nkv, T;
  float eps, q_scale;
  u32 group;                      // tokens of a wave in the values' part (<= STORE_GROUP)
};
#define STORE_GROUP 16u

__device__ __forceinline__ float half_range(float a) {     // saturates at the largest half; NaN stays
  const float r = __builtin_fminf(__builtin_fmaxf(a, -65504.f), 65504.f);
  return a != a ? a : r;
}
__device__ __forceinline__ u32 half_pair(float a, float b) {
  typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
  const half2_t h = {(_Float16)half_range(a), (_Float16)half_range(b)};
  return *(const u32*)&h;
}

// N neighbouring elements in 32 bits (N = 4 or 8; the rows are 16-byte aligned)
template <typename T, int N> __device__ __forceinline__ void load_n(const T* p, float* o);
template <> __device__ __forceinline__ void load_n<float, 4>(const float* p, float* o) { const float4 v = *(const float4*)p; o[0] = v.x; o[1] = v.y; o[2] = v.z; o[3] = v.w; }
template <> __device__ __forceinline__ void load_n<float, 8>(const float* p, float* o) { load_n<float, 4>(p, o); load_n<float, 4>(p + 4, o + 4); }
__device__ __forceinline__ void unpack2(const _Float16*, u32 w, float* o) {
  typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
  const half2_t h = *(const half2_t*)&w;
  o[0] = (float)h[0]; o[1] = (float)h[1];
}
__device__ __forceinline__ void unpack2(const __bf16*, u32 w, float* o) { o[0] = __uint_as_float(w << 16); o[1] = __uint_as_float(w & 0xFFFF0000u); }
// (inputs are read once: non-temporal loads leave the caches to what is written)
template <typename T, int N> __device__ __forceinline__ void load_n(const T* p, float* o) {
  typedef u32 words __attribute__((ext_vector_type(N / 2)));
  const words v = __builtin_nontemporal_load((const words*)p);
#pragma unroll
  for (int i = 0; i < N / 2; ++i) unpack2(p, v[i], o + 2 * i);
}

// scale exponent of a group from the bits of its largest magnitude (fp32): m 2^E -> E - 2, one more from m > 1.75 on, so that the
// largest value is off by half a step at most, in either binade
__device__ __forceinline__ i32 scale_exponent(u32 top) {
  const i32 e = (i32)(top >> 23) - 127 - 2 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return max(KV_E_MIN, min(KV_E_MAX, e));
}
__device__ __forceinline__ i32 scale_exponent(u64 top) {
  const i32 e = (i32)(top >> 52) - 1023 - 2 + ((top & 0xFFFFFFFFFFFFFull) > 0xC000000000000ull ? 1 : 0);
  return max(KV_E_MIN, min(KV_E_MAX, e));
}
// a double to fp32 for the conversion to codes, which rounds to nearest, ties to even: what is not exact gets an odd last bit and so
// stays on its side of every border
__device__ __forceinline__ float odd_float(double x) {
  const float f = (float)fabs(x);
  const double d = (double)f - fabs(x);
  u32 b = __float_as_uint(f);
  if (d > 0.0) b -= 1;
  if (d != 0.0) b |= 1;
  return __builtin_copysignf(__uint_as_float(b), (float)x);
}
template <int SEL> __device__ __forceinline__ u32 codes2(u32 old, float a, float b, float scale) { return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, a, b, scale, SEL); }

// where things of (block, kv head) lie
template <int HD> __device__ __forceinline__ f16_t* k16(const StoreArgs& a, u32 blk, u32 h) { return (f16_t*)a.cache + ((u64)blk * a.nkv + h) * (16 * HD); }
template <int HD> __device__ __forceinline__ f16_t* v16(const StoreArgs& a, u32 blk, u32 h) { return (f16_t*)a.cache + (((u64)a.n_blocks + blk) * a.nkv + h) * (16 * HD); }
template <int HD> __device__ __forceinline__ unsigned char* rec4(const StoreArgs& a, u32 blk, u32 h) { return (unsigned char*)a.cache + ((u64)blk * a.nkv + h) * (17 * HD); }

// One row (a head of a token: of its queries, or KEY of its keys) by HD / (2 N) lanes, a lane with dimensions N j .. N j + N - 1 and
// those hd/2 further: the pairs of its rotation. A lane has one row and 16-byte loads and stores, except for keys on their way to 4 bits, whose
// 64-bit arithmetic takes twice the registers (N = 4).
template <typename T, int HD, int BITS, bool KEY>
struct StoreRow {
  static constexpr int N = KEY && BITS == 4 ? 4 : 8;
  static constexpr u32 LR = HD / (2 * N);
  float x[2 * N], cs[2 * N];
  u32 h, t;
  i32 pos, slot;
  bool live;
  __device__ __forceinline__ void load(const StoreArgs& a, u32 row) {
    const u32 j = threadIdx.x % LR, heads = KEY ? a.nkv : a.nq;
    t = row / heads; h = row % heads;
    live = t < a.T;
    t = min(t, a.T - 1);
    pos = a.pos[t];
    slot = KEY ? a.slot[t] : 0;
    live = live && (u32)pos < a.rows;
    const T* p = KEY ? (const T*)a.k + (u64)t * a.ks + (u64)h * HD : (const T*)a.q + (u64)t * a.qs + (u64)h * HD;
    load_n<T, N>(p + N * j, x);
    load_n<T, N>(p + HD / 2 + N * j, x + N);
    const float* const c = (const float*)(a.tab + (u64)((u32)pos < a.rows ? (u32)pos : 0u) * (HD / 2) + N * j);
    load_n<float, N>(c, cs);
    load_n<float, N>(c + N, cs + N);
  }
  template <typename F>
  __device__ __forceinline__ void turn(const StoreArgs& a, F (&y)[2 * N], const float* gp, F scale) const {
    const u32 j = threadIdx.x % LR;
#pragma unroll
    for (int i = 0; i < 2 * N; ++i) y[i] = (F)x[i];
    if (gp) {
      float g[2 * N];
      load_n<float, N>(gp + N * j, g);
      load_n<float, N>(gp + HD / 2 + N * j, g + N);
      F ss = 0;
#pragma unroll
      for (int i = 0; i < 2 * N; ++i) ss += y[i] * y[i];
#pragma unroll
      for (u32 o = 1; o < LR; o <<= 1) ss += __shfl_xor(ss, (int)o, (int)LR);
      const F ms = ss * (F)(1.0 / HD) + (F)a.eps;
      F r;
      if constexpr (sizeof(F) == 8) r = 1.0 / sqrt(ms);
      else {
        r = 1.0f / sqrtf(ms);
        // (squares of floats and bf16 numbers can leave the range, at both ends: such a row is first divided by the power of two of its largest
        // magnitude 2^e, and eps by 4^e; where that overflows, the row's results are below 2^-64 and zeros as halves)
        if constexpr (!__is_same(T, _Float16)) {
          if (!(ms >= 0x1p-90f && ms < INFINITY)) {
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < 2 * N; ++i) top = fmaxf(top, fabsf(y[i]));
#pragma unroll
            for (u32 o = 1; o < LR; o <<= 1) top = fmaxf(top, __shfl_xor(top, (int)o, (int)LR));
            const i32 e = (i32)(__float_as_uint(top) >> 23) - 127;
            ss = 0;
#pragma unroll
            for (int i = 0; i < 2 * N; ++i) { y[i] = ldexpf(y[i], -e); ss += y[i] * y[i]; }
#pragma unroll
            for (u32 o = 1; o < LR; o <<= 1) ss += __shfl_xor(ss, (int)o, (int)LR);
            r = 1.0f / sqrtf(ss * (1.0f / HD) + ldexpf(a.eps, -2 * e));
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 2 * N; ++i) y[i] = y[i] * r * (F)g[i];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const F p = y[i] * (F)cs[2 * i] - y[i + N] * (F)cs[2 * i + 1], q = y[i + N] * (F)cs[2 * i] + y[i] * (F)cs[2 * i + 1];
      y[i] = p * scale; y[i + N] = q * scale;
    }
  }
  static __device__ __forceinline__ void put(f16_t* o, const float (&y)[2 * N]) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      u32 w[N / 2];
#pragma unroll
      for (int i = 0; i < N / 2; ++i) w[i] = half_pair(y[u * N + 2 * i], y[u * N + 2 * i + 1]);
      if constexpr (N == 8) *(uint4*)(o + u * (HD / 2)) = make_uint4(w[0], w[1], w[2], w[3]);
      else *(uint2*)(o + u * (HD / 2)) = make_uint2(w[0], w[1]);
    }
  }
  __device__ __forceinline__ void store(const StoreArgs& a) const {
    const u32 j = threadIdx.x % LR;
    // (a row is spread over neighbouring lanes of one wave, which agree on every condition here)
    if constexpr (!KEY) {
      float y[2 * N];
      turn<float>(a, y, a.qg, a.q_scale);
      if (live) put(a.qo + (u64)t * a.qos + (u64)h * HD + N * j, y);
      return;
    }
    const bool in = live && slot >= 0 && (u32)slot / 16 < a.n_blocks;
    const u32 blk = in ? (u32)slot / 16 : 0u, off = (u32)slot % 16;
    if constexpr (BITS == 16) {
      float y[2 * N];
      turn<float>(a, y, a.kg, 1.0f);
      if (in) put(k16<HD>(a, blk, h) + off * HD + N * j, y);
    } else {
      double y[2 * N];
      turn<double>(a, y, a.kg, 1.0);
      unsigned char* rec = rec4<HD>(a, blk, h);
      constexpr u32 LG = 32 / N;                 // lanes that hold the 32 dimensions of a group, each half of the row by itself
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        u64 top = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) top = max(top, (u64)__double_as_longlong(y[u * N + i]) & 0x7FFFFFFFFFFFFFFFull);
#pragma unroll
        for (u32 o = 1; o < LG; o <<= 1) top = max(top, (u64)__shfl_xor((unsigned long long)top, (int)o, (int)LG));
        const bool fine = (top >> 52) != 0x7FFull;
        const i32 e = scale_exponent(top);
        const float sc = __uint_as_float((u32)(e + 127) << 23);
        u32 c = codes2<0>(0u, odd_float(y[u * N]), odd_float(y[u * N + 1]), sc);
        c = codes2<1>(c, odd_float(y[u * N + 2]), odd_float(y[u * N + 3]), sc);
        if constexpr (N == 8) {
          c = codes2<2>(c, odd_float(y[u * N + 4]), odd_float(y[u * N + 5]), sc);
          c = codes2<3>(c, odd_float(y[u * N + 6]), odd_float(y[u * N + 7]), sc);
        }
        if (in) {
          unsigned char* o = rec + off * (HD / 2) + u * (HD / 4) + N / 2 * j;
          if constexpr (N == 8) *(u32*)o = fine ? c : 0u;
          else *(uint16_t*)o = fine ? (uint16_t)c : (uint16_t)0;
          if (j % LG == 0) rec[16 * HD + (u * (HD / 64) + j / LG) * 16 + off] = fine ? (unsigned char)(e + 127) : (unsigned char)255;
        }
      }
    }
  }
};

// Values into halves: they lie with the tokens next to each other, so a wave takes up to 16 tokens of a head through LDS and writes
// what fills an aligned run of four places of a block as 8 bytes (four of them are a row of the block, 16 rows a store), the rest
// as single halves.
template <int HD>
struct ValueShared { f16_t v[4][STORE_GROUP][HD + 2]; i32 slot[4][STORE_GROUP + 4]; };
template <typename T, int HD>
__device__ __forceinline__ void store_values16(const StoreArgs& a, ValueShared<HD>& sh, u32 wg) {
  const u32 w = threadIdx.x >> 6, lane = threadIdx.x & 63, item = wg * 4 + w, group = a.group;
  const u32 groups = (a.T + group - 1) / group;
  const bool live = item < groups * a.nkv;
  const u32 h = live ? item % a.nkv : 0u, t0 = live ? item / a.nkv * group : 0u, n = live ? min(group, a.T - t0) : 0u;
  constexpr u32 LR = HD / 8, RP = 64 / LR;       // lanes of a row, rows of a load
  constexpr u32 RUNS = STORE_GROUP / 4;
  i32 sl = -1;
  if (lane < n) {
    sl = a.slot[t0 + lane];
    if (sl < 0 || (u32)sl / 16 >= a.n_blocks || (u32)a.pos[t0 + lane] >= a.rows) sl = -1;
  }
  if (lane < STORE_GROUP + 4) sh.slot[w][lane] = sl;
  for (u32 r = lane / LR; r < n; r += RP) {
    float x[8];
    load_n<T, 8>((const T*)a.v + (u64)(t0 + r) * a.vs + (u64)h * HD + lane % LR * 8, x);
    u32* o = (u32*)&sh.v[w][r][lane % LR * 8];
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = half_pair(x[2 * i], x[2 * i + 1]);
  }
  __syncthreads();
  // tokens at which an aligned run of four places begins, and the tokens that no run takes
  const i32 s1 = sh.slot[w][min(lane + 1, STORE_GROUP + 3u)], s2 = sh.slot[w][min(lane + 2, STORE_GROUP + 3u)], s3 = sh.slot[w][min(lane + 3, STORE_GROUP + 3u)];
  const bool first = sl >= 0 && (sl & 3) == 0 && s1 == sl + 1 && s2 == sl + 2 && s3 == sl + 3;
  const u64 runs = __ballot(first), taken = runs | runs << 1 | runs << 2 | runs << 3, single = __ballot(sl >= 0) & ~taken;
  u64 m8 = runs;
  for (u32 k = lane % RUNS; k; --k) m8 &= m8 - 1; // this lane's run: number lane % RUNS
  if (m8) {
    const u32 t = (u32)__builtin_ctzll(m8), s = (u32)sh.slot[w][t];
    f16_t* o = v16<HD>(a, s / 16, h) + s % 16;
    for (u32 d = lane / RUNS; d < HD; d += 64 / RUNS) {
      const u32 lo = (u32)sh.v[w][t][d] | (u32)sh.v[w][t + 1][d] << 16, hi = (u32)sh.v[w][t + 2][d] | (u32)sh.v[w][t + 3][d] << 16;
      *(uint2*)(o + d * 16) = make_uint2(lo, hi);
    }
  }
  for (u64 m = single; m; m &= m - 1) {
    const u32 t = (u32)__builtin_ctzll(m), s = (u32)sh.slot[w][t];
    f16_t* o = v16<HD>(a, s / 16, h) + s % 16;
    for (u32 d = lane; d < HD; d += 64) o[d * 16] = sh.v[w][t][d];
  }
}

// Values into 4 bits: a lane takes 8 dimensions of a token, four lanes a group.
template <typename T, int HD>
__device__ __forceinline__ void store_values4(const StoreArgs& a, u32 wg) {
  constexpr u32 LR = HD / 8, RPW = 256 / LR;
  const u32 row = wg * RPW + threadIdx.x / LR, t0 = row / a.nkv, h = row % a.nkv, t = min(t0, a.T - 1), j = threadIdx.x % LR;
  const i32 slot = a.slot[t];
  const bool in = t0 < a.T && slot >= 0 && (u32)slot / 16 < a.n_blocks && (u32)a.pos[t] < a.rows;
  float x[8];
  load_n<T, 8>((const T*)a.v + (u64)t * a.vs + (u64)h * HD + 8 * j, x);
  u32 top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
  top = max(top, (u32)__shfl_xor((int)top, 1));
  top = max(top, (u32)__shfl_xor((int)top, 2));
  const bool fine = (top >> 23) != 0xFFu;
  const i32 e = scale_exponent(top);
  const float sc = __uint_as_float((u32)(e + 127) << 23);
  u32 c = codes2<0>(0u, x[0], x[1], sc);
  c = codes2<1>(c, x[2], x[3], sc);
  c = codes2<2>(c, x[4], x[5], sc);
  c = codes2<3>(c, x[6], x[7], sc);
  if (!fine) c = 0;
  if (!in) return;
  const u32 off = (u32)slot % 16;
  unsigned char* rec = rec4<HD>(a, (u32)slot / 16, h);
  if constexpr (HD == 128) {
    *(u32*)(rec + 8 * HD + off / 4 * 256 + j * 16 + off % 4 * 4) = c;
  } else {
    uint16_t* o = (uint16_t*)(rec + 8 * HD + off / 4 * 128 + 2 * j * 8 + off % 4 * 2);
    o[0] = (uint16_t)c; o[4] = (uint16_t)(c >> 16);
  }
  if (j % 4 == 0) rec[16 * HD + HD / 2 + j / 4 * 16 + off] = fine ? (unsigned char)(e + 127) : (unsigned char)255;
}

// tokens of a wave of the values' part: as many as there are when the chip has waves enough, else few, so that there are (64 tokens of 8
// heads: 3.3 us, with 16 a wave 3.8)
__host__ __device__ __forceinline__ u32 store_group(u32 T, u32 nkv, u32 n_cu) {
  u32 g = STORE_GROUP;
  while (g > 4 && (u64)T * nkv / g < 8ull * n_cu) g /= 2;
  return g;
}
// workgroups of the values' part (they come first: theirs are the longer chains) and of the rows' part
__host__ __device__ __forceinline__ u32 store_value_wgs(u32 T, u32 nkv, u32 hd, u32 bits, u32 group) {
  return bits == 16 ? ((T + group - 1) / group * nkv + 3) / 4 : (T * nkv + 2048 / hd - 1) / (2048 / hd);
}
__host__ __device__ __forceinline__ u32 store_key_wgs(u32 T, u32 nkv, u32 hd, u32 bits) {
  const u32 per = (bits == 16 ? 4096 : 2048) / hd;
  return (T * nkv + per - 1) / per;
}
__host__ __device__ __forceinline__ u32 store_query_wgs(u32 T, u32 nq, u32 hd) { return (T * nq + 4096 / hd - 1) / (4096 / hd); }
__host__ __device__ __forceinline__ u32 store_wgs(u32 T, u32 nq, u32 nkv, u32 hd, u32 bits, u32 group) {
  return store_value_wgs(T, nkv, hd, bits, group) + store_key_wgs(T, nkv, hd, bits) + store_query_wgs(T, nq, hd);
}

template <typename T, int HD, int BITS>
__device__ __forceinline__ void kv_store(const StoreArgs& a, ValueShared<HD>& sh, u32 wg) {
  const u32 nv = store_value_wgs(a.T, a.nkv, HD, BITS, a.group), nk = store_key_wgs(a.T, a.nkv, HD, BITS);
  if (wg < nv) {
    if constexpr (BITS == 16) store_values16<T, HD>(a, sh, wg);
    else store_values4<T, HD>(a, wg);
  } else if (wg < nv + nk) {
    StoreRow<T, HD, BITS, true> r;
    r.load(a, (wg - nv) * (256 / r.LR) + threadIdx.x / r.LR);
    r.store(a);
  } else {
    StoreRow<T, HD, BITS, false> r;
    r.load(a, (wg - nv - nk) * (256 / r.LR) + threadIdx.x / r.LR);
    r.store(a);
  }
}

// ---- tokens read back as halves ---------------------------------------------------------------------------------------------
struct ReadArgs {
  const void* cache;
  u32 bits, n_blocks, nkv, T;
  const i32* slot;                // a place outside the cache leaves its rows as they are
  f16_t *ko, *vo;                 // [token][kv head][hd]
};
template <int HD>
__device__ __forceinline__ void kv_read(const ReadArgs& a, u64 i) {      // eight dimensions of a (token, kv head)
  if (i >= (u64)a.T * a.nkv * (HD / 8)) return;
  const u32 j = (u32)(i % (HD / 8)), h = (u32)(i / (HD / 8) % a.nkv), t = (u32)(i / (HD / 8) / a.nkv);
  const i32 slot = a.slot[t];
  if (slot < 0 || (u32)slot / 16 >= a.n_blocks) return;
  const u32 blk = (u32)slot / 16, off = (u32)slot % 16;
  u32 k[4], v[4];
  if (a.bits == 16) {
    const f16_t* kp = (const f16_t*)a.cache + ((u64)blk * a.nkv + h) * (16 * HD) + off * HD + 8 * j;
    const f16_t* vp = (const f16_t*)a.cache + (((u64)a.n_blocks + blk) * a.nkv + h) * (16 * HD) + 8 * j * 16 + off;
    const uint4 x = *(const uint4*)kp;
    k[0] = x.x; k[1] = x.y; k[2] = x.z; k[3] = x.w;
#pragma unroll
    for (int m = 0; m < 4; ++m) v[m] = (u32)vp[2 * m * 16] | (u32)vp[(2 * m + 1) * 16] << 16;
  } else {
    typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
    const unsigned char* rec = (const unsigned char*)a.cache + ((u64)blk * a.nkv + h) * (17 * HD);
    const u32 kc = *(const u32*)(rec + off * (HD / 2) + 4 * j);
    u32 vc;
    if (HD == 128) vc = *(const u32*)(rec + 8 * HD + off / 4 * 256 + j * 16 + off % 4 * 4);
    else {
      const uint16_t* p = (const uint16_t*)(rec + 8 * HD + off / 4 * 128 + 2 * j * 8 + off % 4 * 2);
      vc = (u32)p[0] | (u32)p[4] << 16;
    }
    const float ks = __uint_as_float((u32)rec[16 * HD + j / 4 * 16 + off] << 23), vs = __uint_as_float((u32)rec[16 * HD + HD / 2 + j / 4 * 16 + off] << 23);
    half2_t x[8] = {__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(kc, ks, 0), __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(kc, ks, 1), __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(kc, ks, 2),
                    __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(kc, ks, 3), __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(vc, vs, 0), __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(vc, vs, 1),
                    __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(vc, vs, 2), __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(vc, vs, 3)};
#pragma unroll
    for (int m = 0; m < 4; ++m) { k[m] = *(const u32*)&x[m]; v[m] = *(const u32*)&x[4 + m]; }
  }
  const u64 o = ((u64)t * a.nkv + h) * HD + 8 * j;
  *(uint4*)(a.ko + o) = make_uint4(k[0], k[1], k[2], k[3]);
  *(uint4*)(a.vo + o) = make_uint4(v[0], v[1], v[2], v[3]);
}
