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
// Bound by bytes: each projection is read once, each output written once. What is between is 32-bit arithmetic, with one exception: keys that go
// into 4 bits are normed and rotated in 64 bits, because a sum in another order would move the few values next to a border
// between two codes by half their size. (Values are not computed on: their codes are exact either way.)
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
#define STORE_GROUP 32u

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
template <typename T, int N> __device__ __forceinline__ void load_n(const T* p, float* o) {
  if constexpr (N == 4) {
    const uint2 v = *(const uint2*)p;
    unpack2(p, v.x, o); unpack2(p, v.y, o + 2);
  } else {
    const uint4 v = *(const uint4*)p;
    unpack2(p, v.x, o); unpack2(p, v.y, o + 2); unpack2(p, v.z, o + 4); unpack2(p, v.w, o + 6);
  }
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

// One row (a token's query or key head) by HD/8 lanes, a lane with dimensions 4j .. 4j+3 and hd/2 + 4j .. + 3: the pairs of its rotation.
template <typename T, int HD, int BITS>
struct StoreRow {
  float x[8], g[8];
  float4 cs[2];
  u32 h;
  i32 pos, slot;
  bool live;
  u32 t;
  __device__ __forceinline__ void load(const StoreArgs& a, u32 row, u32 rows) {
    constexpr u32 LR = HD / 8;
    const u32 j = threadIdx.x % LR, heads = a.nq + a.nkv;
    live = row < rows;
    row = min(row, rows - 1);
    t = row / heads; h = row % heads;
    pos = a.pos[t];
    slot = a.slot[t];
    live = live && (u32)pos < a.rows;
    const bool key = h >= a.nq;
    const T* p = key ? (const T*)a.k + (u64)t * a.ks + (u64)(h - a.nq) * HD : (const T*)a.q + (u64)t * a.qs + (u64)h * HD;
    load_n<T, 4>(p + 4 * j, x);
    load_n<T, 4>(p + HD / 2 + 4 * j, x + 4);
    const float4* c = (const float4*)(a.tab + (u64)((u32)pos < a.rows ? (u32)pos : 0u) * (HD / 2) + 4 * j);
    cs[0] = c[0]; cs[1] = c[1];
    const float* gp = key ? a.kg : a.qg;
    if (gp) {
      const float4 lo = *(const float4*)(gp + 4 * j), hi = *(const float4*)(gp + HD / 2 + 4 * j);
      g[0] = lo.x; g[1] = lo.y; g[2] = lo.z; g[3] = lo.w; g[4] = hi.x; g[5] = hi.y; g[6] = hi.z; g[7] = hi.w;
    }
  }
  template <typename F>
  __device__ __forceinline__ void turn(const StoreArgs& a, F (&y)[8], const float* gp, F scale) const {
    constexpr u32 LR = HD / 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (F)x[i];
    if (gp) {
      F ss = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss += y[i] * y[i];
#pragma unroll
      for (u32 o = 1; o < LR; o <<= 1) ss += __shfl_xor(ss, (int)o, (int)LR);
      const F ms = ss * (F)(1.0 / HD) + (F)a.eps;
      F r;
      if constexpr (sizeof(F) == 8) r = 1.0 / sqrt(ms); else r = 1.0f / sqrtf(ms);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = y[i] * r * (F)g[i];
    }
    const float c[4] = {cs[0].x, cs[0].z, cs[1].x, cs[1].z}, s[4] = {cs[0].y, cs[0].w, cs[1].y, cs[1].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const F p = y[i] * (F)c[i] - y[i + 4] * (F)s[i], q = y[i + 4] * (F)c[i] + y[i] * (F)s[i];
      y[i] = p * scale; y[i + 4] = q * scale;
    }
  }
  __device__ __forceinline__ void store(const StoreArgs& a) const {
    constexpr u32 LR = HD / 8;
    const u32 j = threadIdx.x % LR;
    // (a row is spread over neighbouring lanes of one wave, which agree on every condition here)
    if (h < a.nq) {
      float y[8];
      turn<float>(a, y, a.qg, a.q_scale);
      if (live) {
        f16_t* o = a.qo + (u64)t * a.qos + (u64)h * HD + 4 * j;
        *(uint2*)o = make_uint2(half_pair(y[0], y[1]), half_pair(y[2], y[3]));
        *(uint2*)(o + HD / 2) = make_uint2(half_pair(y[4], y[5]), half_pair(y[6], y[7]));
      }
      return;
    }
    const bool in = live && slot >= 0 && (u32)slot / 16 < a.n_blocks;
    const u32 blk = in ? (u32)slot / 16 : 0u, off = (u32)slot % 16;
    if constexpr (BITS == 16) {
      float y[8];
      turn<float>(a, y, a.kg, 1.0f);
      if (in) {
        f16_t* o = k16<HD>(a, blk, h - a.nq) + off * HD + 4 * j;
        *(uint2*)o = make_uint2(half_pair(y[0], y[1]), half_pair(y[2], y[3]));
        *(uint2*)(o + HD / 2) = make_uint2(half_pair(y[4], y[5]), half_pair(y[6], y[7]));
      }
    } else {
      double y[8];
      turn<double>(a, y, a.kg, 1.0);
      u64 top[2] = {0, 0};                       // eight lanes hold the 32 dimensions of a group, each half of the row by itself
#pragma unroll
      for (int i = 0; i < 8; ++i) top[i / 4] = max(top[i / 4], (u64)__double_as_longlong(y[i]) & 0x7FFFFFFFFFFFFFFFull);
#pragma unroll
      for (u32 o = 1; o < 8; o <<= 1) {
        top[0] = max(top[0], (u64)__shfl_xor((unsigned long long)top[0], (int)o, 8));
        top[1] = max(top[1], (u64)__shfl_xor((unsigned long long)top[1], (int)o, 8));
      }
      unsigned char* rec = rec4<HD>(a, blk, h - a.nq);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const bool fine = (top[u] >> 52) != 0x7FFull;
        const i32 e = scale_exponent(top[u]);
        const float sc = __uint_as_float((u32)(e + 127) << 23);
        u32 c = codes2<0>(0u, odd_float(y[4 * u]), odd_float(y[4 * u + 1]), sc);
        c = codes2<1>(c, odd_float(y[4 * u + 2]), odd_float(y[4 * u + 3]), sc);
        if (in) {
          *(uint16_t*)(rec + off * (HD / 2) + u * (HD / 4) + 2 * j) = fine ? (uint16_t)c : (uint16_t)0;
          if (j % 8 == 0) rec[16 * HD + (u * (HD / 64) + j / 8) * 16 + off] = fine ? (unsigned char)(e + 127) : (unsigned char)255;
        }
      }
    }
  }
};

// The rows' part: U rows of a lane group at a time, all loads first.
template <typename T, int HD, int BITS, int U>
__device__ __forceinline__ void store_rows(const StoreArgs& a, u32 wg) {
  constexpr u32 LR = HD / 8, RPW = 256 / LR;
  const u32 rows = a.T * (a.nq + a.nkv), r0 = wg * (RPW * U) + threadIdx.x / LR;
  StoreRow<T, HD, BITS> r[U];
#pragma unroll
  for (int u = 0; u < U; ++u) r[u].load(a, r0 + u * RPW, rows);
#pragma unroll
  for (int u = 0; u < U; ++u) r[u].store(a);
}

// Values into halves: they lie with the tokens next to each other, so a wave takes up to 32 tokens of a head through LDS and writes
// what fills an aligned run of four places of a block as 8 bytes (four of them are a row of the block, 16 rows a store), the rest
// as single halves. Written 2 bytes at a time whatever the places, a prefill's store took as long as all the other stores together.
template <int HD>
struct ValueShared { f16_t v[4][STORE_GROUP][HD + 2]; i32 slot[4][STORE_GROUP + 4]; };
template <typename T, int HD>
__device__ __forceinline__ void store_values16(const StoreArgs& a, ValueShared<HD>& sh, u32 wg) {
  const u32 w = threadIdx.x >> 6, lane = threadIdx.x & 63, item = wg * 4 + w, group = a.group;
  const u32 groups = (a.T + group - 1) / group;
  const bool live = item < groups * a.nkv;
  const u32 h = live ? item % a.nkv : 0u, t0 = live ? item / a.nkv * group : 0u, n = live ? min(group, a.T - t0) : 0u;
  constexpr u32 LR = HD / 8, RP = 64 / LR;       // lanes of a row, rows of a load
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
  for (u32 k = lane % 8; k; --k) m8 &= m8 - 1;   // this lane's run: number lane % 8
  if (m8) {
    const u32 t = (u32)__builtin_ctzll(m8), s = (u32)sh.slot[w][t];
    f16_t* o = v16<HD>(a, s / 16, h) + s % 16;
    for (u32 d = lane / 8; d < HD; d += 8) {
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
  const u32 rows = a.T * a.nkv, row0 = wg * RPW + threadIdx.x / LR, row = min(row0, rows - 1), j = threadIdx.x % LR;
  const u32 t = row / a.nkv, h = row % a.nkv;
  const i32 slot = a.slot[t];
  const bool in = row0 < rows && slot >= 0 && (u32)slot / 16 < a.n_blocks && (u32)a.pos[t] < a.rows;
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

// tokens of a wave of the values' part: as many as there are when the chip has waves enough, else few, so that there are
__host__ __device__ __forceinline__ u32 store_group(u32 T, u32 nkv, u32 n_cu) {
  u32 g = STORE_GROUP;
  while (g > 4 && (u64)T * nkv / g < 8ull * n_cu) g /= 2;
  return g;
}
// workgroups of the values' part (they come first: theirs are the longer chains) and of the rows' part
__host__ __device__ __forceinline__ u32 store_value_wgs(u32 T, u32 nkv, u32 hd, u32 bits, u32 group) {
  return bits == 16 ? ((T + group - 1) / group * nkv + 3) / 4 : (T * nkv + 2048 / hd - 1) / (2048 / hd);
}
__host__ __device__ __forceinline__ u32 store_row_wgs(u32 T, u32 heads, u32 hd, u32 unroll) {
  const u32 per = 2048 / hd * unroll;
  return (T * heads + per - 1) / per;
}

template <typename T, int HD, int BITS, int U>
__device__ __forceinline__ void kv_store(const StoreArgs& a, ValueShared<HD>& sh, u32 wg) {
  const u32 nv = store_value_wgs(a.T, a.nkv, HD, BITS, a.group);
  if (wg < nv) {
    if constexpr (BITS == 16) store_values16<T, HD>(a, sh, wg);
    else store_values4<T, HD>(a, wg);
  } else store_rows<T, HD, BITS, U>(a, wg - nv);
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
