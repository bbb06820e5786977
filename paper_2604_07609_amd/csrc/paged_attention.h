// Attention over the paged cache with a sliding window and first tokens that stay visible, the cache in halves or in 4 bits (layouts:
// kv_store.h). A query at position p sees the keys j <= p of its sequence with j > p - window or j < sinks (window 0: all j <= p).
// A row that sees nothing gives zeros. Softmax in fp32 with a running maximum and sum; the maximum follows only where a score is
// more than 2^8 above it (a probability of up to 256 is a half as exact as one below 1), which spares most tiles the rescale
// and the steps across lanes.
//
// Rows of a sequence and kv head are its queries times the G query heads that share the head: row = query * G + head. Sixteen of
// them are the columns of the matrix products S[key][row] = K q and O^T[dim][row] = V^T P^T; the accumulator of S (column = lane % 16, keys
// 4 (lane / 16) + i) is the operand P^T as it stands. With a 4-bit cache few rows' scores are products of the codes themselves
// (v_mfma_scale_f32_16x16x128_f8f6f4, which takes a scale per 32 of them as they are stored): the query is the sum of three e4m3
// numbers of four bits each, with a scale per 32 dimensions as well: exactly, or (below 2^-14 of the largest of those 32) to within 2^-25 of that
// largest. So three such products give in 32 bits what one with converted keys would, and the vector instructions that
// converted them, which bound the kernel, are gone. Of the values a lane holds 8 neighbouring dimensions of 4 keys, so a register
// pair of the converted values is two dimensions of one key, and each of the two products that take it has zeros for the other
// one's dimension in its P: twice the matrix instructions, which decode has to spare, in place of exchanging halves between registers,
// which it has not.
#pragma once
#include "attention_mfma.h"
#include "kv_store.h"
#include "paged_views.h"

typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef i32 i32x8_t __attribute__((ext_vector_type(8)));
__device__ __forceinline__ u32 f16x2_bits(f16x2_t v) { return *(const u32*)&v; }
__device__ __forceinline__ f16x8_t f16x8_of(u32 a, u32 b, u32 c, u32 d) { const uint4 v = make_uint4(a, b, c, d); return *(const f16x8_t*)&v; }
// Values that are not finite, where some row of the tile must not see them (0 times one would not be 0): the products take the largest finite
// ones in their place (only_finite; where a row does see them, what is added next swallows those), and a product of strange_codes with the
// mask (1 where a row sees a key) tells per row and dimension what it sees: 1 for every +inf, 64 for every -inf, both for NaN (exact: at
// most 32 keys a product). Tiles that no mask touches need none of it.
__device__ __forceinline__ u32 only_finite(u32 w) {
  const f16x2_t top = {(_Float16)65504.f, (_Float16)65504.f};
  return f16x2_bits(__builtin_elementwise_max(__builtin_elementwise_min(*(const f16x2_t*)&w, top), -top));      // (of a number and NaN: the number)
}
__device__ __forceinline__ u32 strange_codes(u32 w) {
  auto one = [&](u32 h) { return (h & 0x7C00u) != 0x7C00u ? 0u : (h & 0x3FFu) ? 0x5410u : h >> 15 ? 0x5400u : 0x3C00u; };      // 65, 64, 1
  return one(w & 0xFFFFu) | one(w >> 16) << 16;
}
__device__ __forceinline__ float strange_sum(float n) {
  const float neg = floorf(n * (1.0f / 64.0f)), pos = n - 64.0f * neg;
  return (pos > 0.f ? INFINITY : 0.f) + (neg > 0.f ? -INFINITY : 0.f);
}
__device__ __forceinline__ bool any_nan(const floatx4_t& z) { return __ballot(z[0] != 0.f || z[1] != 0.f || z[2] != 0.f || z[3] != 0.f) != 0; }
// bit i: the row at position p (-1: no row) sees the key k + i, i < 8
__device__ __forceinline__ u32 sees(const PagedArgs& a, i32 p, i32 k) {
  auto below = [](i32 n) { return (1u << (u32)max(0, min(8, n))) - 1u; };
  u32 seen = below(p + 1 - k);
  if (a.window) seen &= ~below(p + 1 - (i32)a.window - k) | below((i32)a.sinks - k);
  return seen;
}

// ---- few rows: decoding sequences, drafted tokens --------------------------------------------------------------------------
// A wave's tile: 16 keys and values of a kv head.
// A lane's offsets in a tile, as numbers the compiler cannot take apart: it would keep each of their parts as 64-bit addresses, in registers
// that the loop has no room for, where a uniform base and 32 bits per lane are all that a load takes.
template <int HD, int BITS> struct CacheTile;
struct TileLane { u32 k, v, ks, vs; };
__device__ __forceinline__ u32 opaque(u32 x) { asm volatile("" : "+v"(x)); return x; }
typedef u32 u32x4_t __attribute__((ext_vector_type(4)));
typedef u32 u32x2_t __attribute__((ext_vector_type(2)));
typedef const __attribute__((address_space(1))) unsigned char global_byte;
template <typename T> __device__ __forceinline__ T from_global(global_byte* p) { return *(const __attribute__((address_space(1))) T*)p; }
__device__ __forceinline__ global_byte* uniform_global(const void* p) { return (global_byte*)(u64)uniform_ptr((const unsigned char*)p); }
template <int HD>
struct CacheTile<HD, 16> {
  f16x8_t k[HD / 32];
  uint2 v[HD / 16];
  static __device__ __forceinline__ TileLane lane_offsets() {
    const u32 lane = threadIdx.x & 63, lg = lane >> 4, lc = lane & 15;
    return {opaque(lc * (2 * HD) + lg * 16), opaque(lc * 32 + lg * 8), 0, 0};
  }
  __device__ __forceinline__ void load(const PagedArgs& a, const TileLane& at, u32 id, u32 g) {
    const f16_t* const first = (const f16_t*)a.cache + ((u64)id * a.nkv + g) * (16 * HD);
    global_byte *const kp = uniform_global(first), *const vp = uniform_global(first + (u64)a.n_blocks * a.nkv * (16 * HD));
#pragma unroll
    for (int s = 0; s < HD / 32; ++s) { const u32x4_t x = from_global<u32x4_t>(kp + at.k + s * 64); k[s] = *(const f16x8_t*)&x; }
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) { const u32x2_t x = from_global<u32x2_t>(vp + at.v + d * 512); v[d] = make_uint2(x[0], x[1]); }
  }
  struct Query { f16x8_t q[HD / 32]; };
  static __device__ __forceinline__ void load_query(const f16_t* row, Query& r) {
    const u32 lg = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int s = 0; s < HD / 32; ++s) r.q[s] = ld_tile(row + s * 32 + lg * 8);
  }
  __device__ __forceinline__ floatx4_t scores(const Query& r) const {
    floatx4_t x = floatx4_t{0.f, 0.f, 0.f, 0.f}, y = x;              // two chains
#pragma unroll
    for (int s = 0; s < HD / 32; s += 2) {
      x = __builtin_amdgcn_mfma_f32_16x16x32_f16(k[s], r.q[s], x, 0, 0, 0);
      y = __builtin_amdgcn_mfma_f32_16x16x32_f16(k[s + 1], r.q[s + 1], y, 0, 0, 0);
    }
    return x + y;
  }
  struct Probs { f16x4_t p; };
  static __device__ __forceinline__ Probs probs(const float (&p)[4]) { return {f16x4_t{(_Float16)p[0], (_Float16)p[1], (_Float16)p[2], (_Float16)p[3]}}; }
  struct Operand { u32 w[2]; };                                      // values of 16 dimensions
  static constexpr int NV = HD / 16;                                 // operands of a tile's values
  __device__ __forceinline__ Operand operand(int i) const { return {{v[i].x, v[i].y}}; }
  static __device__ __forceinline__ constexpr int of(int d) { return d; }          // operand of the dimensions' tile d
  static __device__ __forceinline__ floatx4_t product(const Operand& x, const Probs& p, int, const floatx4_t& o) {
    const uint2 w = make_uint2(x.w[0], x.w[1]);
    return __builtin_amdgcn_mfma_f32_16x16x16f16(*(const f16x4_t*)&w, p.p, o, 0, 0, 0);
  }
  // whether some value is not finite (then those are taken out); vis: bits of the lane's four keys, seen by the lane's rows
  __device__ __forceinline__ bool take_strange_out(u32) {
    const float zero[4] = {0.f, 0.f, 0.f, 0.f};
    const Probs none = probs(zero);
    floatx4_t z = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) z = product(operand(d), none, 0, z);       // 0 unless something is not finite
    if (!any_nan(z)) return false;
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) v[d] = make_uint2(only_finite(v[d].x), only_finite(v[d].y));
    return true;
  }
  // the 4 dimensions of accumulator tile d, or 4 of the 8 (or 4) neighbouring ones: register i of tile d is dimension
  static __device__ __forceinline__ u32 o_dim(int d, u32 lg, int i) { return d * 16 + lg * 4 + i; }
};
template <int HD>
struct CacheTile<HD, 4> {
  u32 k[4];                       // 32 dimensions of a key: lane % 16, dimensions 32 (lane / 16) .. (heads of 64: of lane / 16 % 2)
  u32 v[HD / 32];                 // HD / 16 dimensions of 4 values
  u32 ks, vs;                     // scale of the key's dimensions; of the 4 values'
  static __device__ __forceinline__ TileLane lane_offsets() {
    const u32 lane = threadIdx.x & 63, lg = lane >> 4, lc = lane & 15, kg = lg % (HD / 32);
    return {opaque(lc * (HD / 2) + kg * 16), opaque((lg * 16 + lc) * (HD / 8)), opaque(kg * 16 + lc), opaque(lc / (HD == 128 ? 4 : 8) * 16 + lg * 4)};
  }
  __device__ __forceinline__ void load(const PagedArgs& a, const TileLane& at, u32 id, u32 g) {
    global_byte* const r = uniform_global((const unsigned char*)a.cache + ((u64)id * a.nkv + g) * (17 * HD));
    const u32x4_t x = from_global<u32x4_t>(r + at.k);
    k[0] = x[0]; k[1] = x[1]; k[2] = x[2]; k[3] = x[3];
    if constexpr (HD == 128) {
      const u32x4_t y = from_global<u32x4_t>(r + at.v + 8 * HD);
      v[0] = y[0]; v[1] = y[1]; v[2] = y[2]; v[3] = y[3];
    } else {
      const u32x2_t y = from_global<u32x2_t>(r + at.v + 8 * HD);
      v[0] = y[0]; v[1] = y[1];
    }
    ks = *(r + at.ks + 16 * HD);
    vs = from_global<u32>(r + at.vs + (16 * HD + HD / 2));
  }
  // The product's B operand holds the elements 16 g .. and 64 + 16 g .. of its 128 in lane group g, its scales (like A's) are those of the
  // elements 32 g .. in lane group g. Parts: with the largest magnitude of 32 dimensions (those that share a scale, as a key's do) in
  // [128, 256), e4m3(x), e4m3(16 (x - that)) and so on: each takes four bits off a half's eleven, down to 2^-25 of that largest. Heads of
  // 64: A holds a key's codes twice, and the second part meets the upper ones.
  static constexpr int NP = HD == 128 ? 3 : 2;
  struct Query { i32x8_t part[NP]; u32 scale; };     // scale: byte i for product i
  static __device__ __forceinline__ void load_query(const f16_t* row, Query& r) {
    const u32 lg = (threadIdx.x & 63) >> 4;
    float x[HD / 4];
#pragma unroll
    for (int h = 0; h < HD / 64; ++h)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const f16x8_t y = ld_tile(row + h * 64 + lg * 16 + i * 8);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[h * 16 + i * 8 + j] = (float)y[j];
      }
    u32 scale[HD / 64];                                              // of the lane's 16 of the dimensions 64 h .., which two lane groups share
#pragma unroll
    for (int h = 0; h < HD / 64; ++h) {
      u32 top = 0;
#pragma unroll
      for (int i = h * 16; i < h * 16 + 16; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
      top = max(top, (u32)__shfl_xor((int)top, 16));
      const bool fine = top < 0x7F800000u;
      const i32 e = top ? (i32)(top >> 23) - 127 - 7 : 0;            // (a half is a normal float)
      const float up = __uint_as_float((u32)(127 - (fine ? e : 0)) << 23);
#pragma unroll
      for (int i = h * 16; i < h * 16 + 16; ++i) x[i] = fine ? x[i] * up : 0.f;
      scale[h] = fine ? (u32)(127 + e) : 255u;                       // (with an infinity or NaN: the row's scores are not a number)
    }
    i32 part[4][HD / 16] = {};
#pragma unroll
    for (int p = 0; p < 3; ++p) {
#pragma unroll
      for (int j = 0; j < HD / 16; ++j) {
        i32 w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * j], x[4 * j + 1], 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * j + 2], x[4 * j + 3], w, true);
        part[p][j] = w;
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
        x[4 * j] = (x[4 * j] - lo[0]) * 16.f; x[4 * j + 1] = (x[4 * j + 1] - lo[1]) * 16.f;
        x[4 * j + 2] = (x[4 * j + 2] - hi[0]) * 16.f; x[4 * j + 3] = (x[4 * j + 3] - hi[1]) * 16.f;
      }
    }
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int j = 0; j < 8; ++j) r.part[p][j] = HD == 128 ? part[p][j] : part[2 * p + j / 4][j % (HD / 16)];
    // the scale that this lane group gives: that of dimensions 32 lg .. (heads of 64: 32 (lg % 2) .., of the second part where lg / 2)
    const int from = (int)((lg & 1) * 32 + (threadIdx.x & 15));
    u32 s0 = (u32)__shfl((int)scale[0], from);
    if constexpr (HD == 128) { const u32 s1 = (u32)__shfl((int)scale[1], from); s0 = lg >= 2 ? s1 : s0; }
    const bool fine = s0 != 255;
    if (HD == 64 && lg >= 2) s0 -= 4;
    r.scale = !fine ? 0xFFFFFFu : HD == 128 ? s0 | (s0 - 4) << 8 | (s0 - 8) << 16 : s0 | (s0 - 8) << 8;
  }
  __device__ __forceinline__ floatx4_t scores(const Query& r) const {
    const i32x8_t a = {(i32)k[0], (i32)k[1], (i32)k[2], (i32)k[3], 0, 0, 0, 0};
    floatx4_t x = floatx4_t{0.f, 0.f, 0.f, 0.f};                     // (formats: A e2m1 = 4, B e4m3 = 0)
    x = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, r.part[0], x, 4, 0, 0, (i32)ks, 0, (i32)r.scale);
    x = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, r.part[1], x, 4, 0, 0, (i32)ks, 1, (i32)r.scale);
    if constexpr (NP == 3) x = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, r.part[NP - 1], x, 4, 0, 0, (i32)ks, 2, (i32)r.scale);
    return x;
  }
  struct Probs { f16x8_t even, odd; };                               // the probability at the lower, at the upper half of each word
  static __device__ __forceinline__ Probs probs(const float (&p)[4]) {
    u32 e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) { const _Float16 h = (_Float16)p[i]; e[i] = *(const uint16_t*)&h; }
    return {f16x8_of(e[0], e[1], e[2], e[3]), f16x8_of(e[0] << 16, e[1] << 16, e[2] << 16, e[3] << 16)};
  }
  struct Operand { u32 w[4]; };                                      // a pair of dimensions' tiles, of 4 values
  static constexpr int NV = HD / 32;
  __device__ __forceinline__ Operand operand(int i) const {
    Operand r;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const float sc = __uint_as_float((vs >> (8 * t) & 0xFFu) << 23);
      const u32 w = HD == 128 ? v[t] : t & 1 ? v[t / 2] >> 16 : v[t / 2];
      r.w[t] = f16x2_bits(i == 0 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, sc, 0) : i == 1 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, sc, 1)
                        : i == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, sc, 2) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, sc, 3));
    }
    return r;
  }
  static __device__ __forceinline__ constexpr int of(int d) { return d / 2; }
  static __device__ __forceinline__ floatx4_t product(const Operand& x, const Probs& p, int d, const floatx4_t& o) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(f16x8_of(x.w[0], x.w[1], x.w[2], x.w[3]), d & 1 ? p.odd : p.even, o, 0, 0, 0);
  }
  // (Keys that no row sees, in places that may hold anything, become zeros. With scales from 141 on values leave the halves, and 255 is
  // not a number: the other scales give finite ones.)
  __device__ __forceinline__ bool take_strange_out(u32 vis) {
    vis |= (u32)__builtin_amdgcn_update_dpp(0, (i32)vis, 0x128, 0xF, 0xF, false);      // the 16 lanes of the same keys: row_ror 8, 4, 2, 1
    vis |= (u32)__builtin_amdgcn_update_dpp(0, (i32)vis, 0x124, 0xF, 0xF, false);
    vis |= (u32)__builtin_amdgcn_update_dpp(0, (i32)vis, 0x122, 0xF, 0xF, false);
    vis |= (u32)__builtin_amdgcn_update_dpp(0, (i32)vis, 0x121, 0xF, 0xF, false);
    vs &= ((vis & 15u) * 0x00204081u & 0x01010101u) * 0xFFu;
    const u32 odd = ((vs & 0x7F7F7F7Fu) + (0x80u - KV_E_MAX) * 0x01010101u) & vs & 0x80808080u;      // from 128 + KV_E_MAX on
    if (!__ballot(odd != 0)) return false;
    vs &= ~((odd >> 7) * 0xFFu);
    return true;
  }
  static __device__ __forceinline__ u32 o_dim(int d, u32 lg, int i) { return (lg * 4 + i) * (HD / 16) + d; }
};

#define PAGED_WAVES 8              // waves of a workgroup of the prompt part
struct NoLinks {};
struct ViewLinks { uint16_t link[PAGED_MAX_SEQS]; };      // of a sequence: its group, or NO_GROUP; of a group: the sequence whose table it takes
template <int HD, int CT, int NW, bool SHARED = false>
struct ShortShared : std::conditional<SHARED, ViewLinks, NoLinks>::type {
  // a result that one wave leaves for others, as its registers hold it: of the pair that its run begins inside of; at NW, of the pair
  // that goes on in other workgroups, by the wave that it begins in
  floatx4_t o[NW + 1][CT][HD / 16][64];
  float m[NW + 1][CT][16], l[NW + 1][CT][16];
  u32 pre[PAGED_MAX_SEQS + 1], wave_sum[NW], last[2], need[2];      // need: results of the pair, last: this is the last one
  u32* ctr[2];
  i32 pos0[PAGED_MAX_SEQS];
  unsigned char n[PAGED_MAX_SEQS];                   // (a short sequence has at most 64 rows)
};

__device__ __forceinline__ u32 wave_sums(u32 v) {     // inclusive prefix sums over the wave
  const u32 lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) { const u32 x = __shfl_up(v, o); if (lane >= (u32)o) v += x; }
  return v;
}
// exclusive prefix sums of f(0 .. n) into pre[0 .. n], by a workgroup of NW waves
template <u32 NW, typename F>
__device__ __forceinline__ void prefix_sums(u32* pre, u32* wave_sum, u32 n, F f) {
  const u32 lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  u32 base = 0;
  for (u32 i0 = 0; i0 < n; i0 += 64 * NW) {
    const u32 i = i0 + threadIdx.x;
    const u32 v = wave_sums(i < n ? f(i) : 0u);
    __syncthreads();
    if (lane == 63) wave_sum[w] = v;
    __syncthreads();
    u32 before = base;
    for (u32 k = 0; k < NW; ++k) { if (k < w) before += wave_sum[k]; base += wave_sum[k]; }
    if (i < n) pre[i + 1] = before + v;
  }
  if (threadIdx.x == 0) pre[0] = 0;
  __syncthreads();
}
// last s < n (at most PAGED_MAX_SEQS) with pre[s] <= x, x the same in the whole wave, whose lanes look at 64 places at a time (two
// readings of LDS one after the other, and not ten)
__device__ __forceinline__ u32 last_at_most(const u32* pre, u32 n, u32 x) {
  if (n == 1) return 0;
  const u32 lane = threadIdx.x & 63, step = (n + 63) / 64;
  auto below = [&](u32 i, u32 end) { return (u32)__popcll(__ballot(i < end && pre[i < end ? i : 0u] <= x)); };
  const u32 lo = (below(lane * step, n) - 1) * step;
  return lo + below(lo + lane, min(lo + step, n)) - 1;
}

// running maximum, sum and output of one tile of 16 rows, and one tile of keys and values added to them
template <int HD, int BITS>
struct ShortAcc {
  typedef CacheTile<HD, BITS> Tile;
  floatx4_t o[HD / 16];
  float m, l;
  __device__ __forceinline__ void init() {
    m = -INFINITY; l = 0.f;
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) o[d] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  }
  // maximum and sum with another result's; the factors of this one's output and of the other's
  __device__ __forceinline__ void join(float m2, float l2, float& mine, float& other) {
    const float mn = fmaxf(m, m2), ref = mn == -INFINITY ? 0.f : mn;
    mine = __builtin_amdgcn_exp2f(m - ref); other = __builtin_amdgcn_exp2f(m2 - ref);
    l = l * mine + l2 * other;
    m = mn;
  }
  // vis: bit i of the lane's four keys seen by the lane's row (used where `edge`)
  __device__ __forceinline__ void add(const Tile& t, const typename Tile::Query& q, float c, bool edge, u32 vis) {
    floatx4_t s = t.scores(q);
    if (edge) {
      asm volatile("" ::: "memory");                                 // (a branch: few tiles are)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = vis >> i & 1u ? s[i] : -INFINITY;
    }
    float top = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])) * c;
    if (__ballot(top > m + 8.f)) {
      top = quad_max(top);
      const float mn = fmaxf(m, top);
      const float f = mn == m || m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);      // (nothing yet but an infinity, maybe: not times 0)
      l *= f;
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) o[d] *= f;
      m = mn;
    }
    const float ref = m == -INFINITY ? 0.f : -m;
    float p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) { p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, ref)); l += p[i]; }      // exp2(-inf) = 0
    const typename Tile::Probs pp = Tile::probs(p);
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) o[d] = Tile::product(t.operand(Tile::of(d)), pp, d, o[d]);
  }
};
template <int HD, int BITS, int CT, int NW, typename Shared>
__device__ __forceinline__ void leave_in_lds(Shared& sh, u32 at, const ShortAcc<HD, BITS> (&acc)[CT]) {
  const u32 lane = threadIdx.x & 63;
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const float l = quad_sum(acc[c].l);
    if (lane < 16) { sh.m[at][c][lane] = acc[c].m; sh.l[at][c][lane] = l; }
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) sh.o[at][c][d][lane] = acc[c].o[d];
  }
}
template <int HD, int BITS, int CT, int NW, typename Shared>
__device__ __forceinline__ void add_from_lds(const Shared& sh, u32 at, ShortAcc<HD, BITS> (&acc)[CT]) {
  const u32 lane = threadIdx.x & 63;
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    float mine, other;
    acc[c].join(sh.m[at][c][lane & 15], lane < 16 ? sh.l[at][c][lane] : 0.f, mine, other);       // (a sum is that of the row's four lanes)
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) acc[c].o[d] = acc[c].o[d] * mine + sh.o[at][c][d][lane] * other;
  }
}
// a result in global memory, for another workgroup (see merge_chunks for why past the caches): maxima, sums, outputs as registers hold them
template <int HD, int CT> __device__ __forceinline__ constexpr u32 short_slot() { return CT * (128 + HD * 16); }     // floats
// A result in LDS or in the workspace: the lane's maximum and sum of a row tile, its tile d of dimensions
template <typename Shared>
struct LdsResult {
  const Shared& sh;
  u32 at;
  __device__ __forceinline__ float m(u32 c, u32 lane) const { return sh.m[at][c][lane & 15]; }
  __device__ __forceinline__ float l(u32 c, u32 lane) const { return lane < 16 ? sh.l[at][c][lane] : 0.f; }       // (the row's four lanes' added up)
  __device__ __forceinline__ floatx4_t o(u32 c, u32 d, u32 lane) const { return sh.o[at][c][d][lane]; }
};
template <int HD>
struct FarResult {
  const float* p;
  __device__ __forceinline__ float m(u32 c, u32 lane) const { return ld_past_caches(p + c * (128 + HD * 16) + lane); }
  __device__ __forceinline__ float l(u32 c, u32 lane) const { return ld_past_caches(p + c * (128 + HD * 16) + 64 + lane); }
  __device__ __forceinline__ floatx4_t o(u32 c, u32 d, u32 lane) const {
    const u64* const q = (const u64*)(p + c * (128 + HD * 16) + 128 + (d * 64 + lane) * 4);
    const u64 x = __hip_atomic_load(q, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), y = __hip_atomic_load(q + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return floatx4_t{__uint_as_float((u32)x), __uint_as_float((u32)(x >> 32)), __uint_as_float((u32)y), __uint_as_float((u32)(y >> 32))};
  }
};
// Results added up by a whole workgroup: a wave has T of the tiles of dimensions, of all results, and asks for those of eight results at a
// time. (A wave with all dimensions of every NWth result, one after the other, took three times as long.)
template <int HD, int BITS, int CT, int NW>
struct ShortMerge {
  static constexpr int TILES = CT * (HD / 16), T = TILES > NW ? TILES / NW : 1, AT_ONCE = 8;
  u32 c, d0;                                         // row tile, first tile of dimensions
  bool live;                                         // the lane has a row, the wave tiles
  floatx4_t o[T];
  float m, l;
  template <typename F>
  __device__ __forceinline__ void sum(u32 x0, u32 x1, u32 rows, F result) {      // results x0 .. x1
    const u32 lane = threadIdx.x & 63, w = (u32)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    c = w * T / (HD / 16); d0 = w * T % (HD / 16);
    live = w * T < (u32)TILES && c * 16 + (lane & 15) < rows;
    m = -INFINITY; l = 0.f;
#pragma unroll
    for (int t = 0; t < T; ++t) o[t] = floatx4_t{0.f, 0.f, 0.f, 0.f};
    if (!live) return;
#pragma unroll 1
    for (u32 x = x0; x < x1; x += AT_ONCE) {
      float ms[AT_ONCE], ls[AT_ONCE];
      floatx4_t v[AT_ONCE][T];
#pragma unroll
      for (int b = 0; b < AT_ONCE; ++b) {
        ms[b] = -INFINITY; ls[b] = 0.f;
#pragma unroll
        for (int t = 0; t < T; ++t) v[b][t] = floatx4_t{0.f, 0.f, 0.f, 0.f};
        if (x + b < x1) {
          const auto r = result(x + b);
          ms[b] = r.m(c, lane); ls[b] = r.l(c, lane);
#pragma unroll
          for (int t = 0; t < T; ++t) v[b][t] = r.o(c, d0 + t, lane);
        }
      }
      float mn = m;
#pragma unroll
      for (int b = 0; b < AT_ONCE; ++b) mn = fmaxf(mn, ms[b]);
      const float ref = mn == -INFINITY ? 0.f : mn, f = __builtin_amdgcn_exp2f(m - ref);
      l *= f;
#pragma unroll
      for (int t = 0; t < T; ++t) o[t] *= f;
#pragma unroll
      for (int b = 0; b < AT_ONCE; ++b) {
        const float g = __builtin_amdgcn_exp2f(ms[b] - ref);
        l += ls[b] * g;
#pragma unroll
        for (int t = 0; t < T; ++t) o[t] += v[b][t] * g;
      }
      m = mn;
    }
  }
  // into the workspace (see merge_chunks for why past the caches)
  __device__ __forceinline__ void leave(float* result) const {
    const u32 lane = threadIdx.x & 63;
    if (!live) return;
    float* const p = result + c * (128 + HD * 16);
    if (d0 == 0) { st_past_caches(p + lane, m); st_past_caches(p + 64 + lane, l); }
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        __hip_atomic_store((u64*)(p + 128 + ((d0 + t) * 64 + lane) * 4) + h, ((u64)__float_as_uint(o[t][2 * h + 1]) << 32) | __float_as_uint(o[t][2 * h]), __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
  }
};
// What CacheTile::take_strange_out has taken out of a tile, given to the rows that see it (vis: bits of the lane's four keys). Rare, and
// so one step after the other: there are no registers for it.
template <int HD, int BITS>
__device__ __forceinline__ void give_strange(const CacheTile<HD, BITS>& t, floatx4_t (&o)[HD / 16], u32 vis) {
  typedef CacheTile<HD, BITS> Tile;
  constexpr int PER = HD / 16 / Tile::NV;            // tiles of dimensions per operand
  const float see[4] = {vis & 1u ? 1.f : 0.f, vis & 2u ? 1.f : 0.f, vis & 4u ? 1.f : 0.f, vis & 8u ? 1.f : 0.f};
  const typename Tile::Probs p = Tile::probs(see);
#pragma unroll
  for (int v = 0; v < Tile::NV; ++v) {
    typename Tile::Operand x = t.operand(v);
#pragma unroll
    for (u32& w : x.w) w = strange_codes(w);
#pragma unroll
    for (int d = v * PER; d < (v + 1) * PER; ++d) {
      const floatx4_t n = Tile::product(x, p, d, floatx4_t{0.f, 0.f, 0.f, 0.f});
#pragma unroll
      for (int i = 0; i < 4; ++i) o[d][i] += strange_sum(n[i]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}

// whether a view's results are joined with others
template <typename Shared>
__device__ __forceinline__ bool is_joined(const SharedArgs& a, const Shared& sh, u32 s) { return s >= a.n_seqs || (u32)__builtin_amdgcn_readfirstlane(sh.link[s]) != NO_GROUP; }
// The kernel's arguments (its first and only ones), loaded anew: each part of the kernel has its own copy, or the compiler would load them once at the
// start, and keep what is more than the scalar registers hold in vector registers, to be brought back at every tile.
__device__ __forceinline__ SharedArgs fresh_args() {
  typedef const __attribute__((address_space(4))) SharedArgs* args_t;
  u64 p = (u64)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const SharedArgs*)(args_t)p;
}
// a row's result, to be joined with another one (which: 0 the group's, 1 the sequence's)
template <int HD>
__device__ __forceinline__ float* row_result(const SharedArgs& a, u32 which, u32 row, u32 head) {
  return a.rows + (((u64)which * a.n_rows + row) * a.nq + head) * ROW_RESULT(HD);
}
// of query k (row_index), with the arguments loaded anew: they would take registers that the loops need (4 sequences: 20.9 us, so 20.5)
template <int HD>
__device__ __forceinline__ float* row_result(u32 which, u32 s, u32 t0, u32 k, u32 head) {
  const SharedArgs a = fresh_args();
  return row_result<HD>(a, which, row_index(a, s, t0, k), head);
}

__device__ __forceinline__ f16_t* out_at(const PagedArgs& a, u32 tok, u32 k) { return a.out_tbs ? a.out + packed_off(tok, k, a.out_tbs) : a.out + (u64)tok * a.os + k; }

// Bound by bytes where there are many: 256 sequences of up to 1028 visible keys (8 kv heads of 128, halves) 574 MB in 122 us, 4.7 TB/s,
// 1.05 GB of long contexts 5.6; 128 sequences of 3000 to 16384 in 4 bits 1.10 GB in 209 us, 5.3 TB/s. What is left of
// 6.3 is the start (7 us to the first tile: lengths, ids, tile, one after the other), the end (8 us: a workgroup's results joined and
// handed on) and XCDs that are up to a tenth slower than others, another one in every launch. Few keys are bound by those latencies.
//
// All tiles of all (sequence, kv head) pairs are one line of units, cut into equal runs, one per wave: whatever the lengths, every
// wave reads the same number of bytes, with NT tiles on their way, and waits for nobody until its run ends.
// A pair inside a run is finished where it is. One that several waves of a workgroup share is added up by the wave it begins in (in
// LDS, after the one barrier); of one that several workgroups share, each adds up its waves' results and leaves one in the
// workspace, and the workgroup that comes last adds those up, its waves a part of the dimensions each. Of more than SHORT_GROUP such
// results, those of every SHORT_GROUP workgroups are added up by the last of these first: of one sequence of 65531 keys in 4
// bits, 128 results a pair, 53 us in one go, 24 in groups of 16 or 8; of 16384 keys, 32 results, 20.6, 18.1 and 16.3. All sums in the
// order of the runs: results do not depend on who comes when.
// Few short pairs (half as many as workgroups) are dealt out whole instead, a workgroup or several to each, 32 to 64 tiles a
// workgroup: 3 sequences of 100 keys 8.4 us and not 18, 12 of 1500 20 and not 23, 48 x 5 drafted tokens 20 and not 26. With up to 32 tiles one
// workgroup has a pair for itself: two, of 16 sequences of 500 keys in 4 bits, take 12.0 us in place of 11.3.
// The loop over tiles is written out NT times for its registers, so all that is rare stands outside of it, once.
#define SHORT_GROUP 8u
// 32-bit counters of a launch of nwg workgroups and floats of its results. The counters: two for the prompt part, one per workgroup (of the
// pair that begins in it and goes on in others: one at most), two per group. They do not depend on the batch.
__host__ __device__ __forceinline__ u32 paged_counters(u32 nwg) { return 2 + nwg + 2 * ((nwg + SHORT_GROUP - 1) / SHORT_GROUP); }
__host__ __device__ __forceinline__ u64 short_floats(u32 nwg, u32 hd, u32 ct) { return 2ull * (nwg + (nwg + SHORT_GROUP - 1) / SHORT_GROUP) * ct * (128 + 16 * hd); }
template <int HD, int BITS, int CT, int NT, int NW, typename A>
__device__ __forceinline__ void paged_short(const A& a, ShortShared<HD, CT, NW, is_shared<A>>& sh, u32 wg, u32 nwg) {
  typedef ShortShared<HD, CT, NW, is_shared<A>> Shared;
  constexpr bool SHARED = is_shared<A>;
  // Units ahead of a pair's that are no tiles, but what the pair takes besides: where most pairs are of a tile or two, and some long, runs of as many tiles
  // were up to twice as long as others (40 groups of up to four sequences with 9 tokens of their own: 58 us the longest, 34 half of them)
  constexpr u32 GAP = SHARED ? FEW_PAIR : 0u;
  typedef CacheTile<HD, BITS> Tile;
  const u32 lane = threadIdx.x & 63, w = (u32)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lg = lane >> 4, lc = lane & 15;
  auto scalar = [](u32 x) { return (u32)__builtin_amdgcn_readfirstlane(x); };
  // of a view: position of the last query, first key (only where there are groups is it another one than of a sequence's own)
  auto last_pos = [&](u32 s, i32 p0, i32 n) { return p0 + (SHARED && s >= a.n_seqs ? 1 : n) - 1; };
  auto first_key = [&](u32 s) {
    if constexpr (SHARED) return s < a.n_seqs && sh.link[s] != NO_GROUP ? (u32)sh.pos0[a.n_seqs + sh.link[s]] + 1 : 0u;
    return 0u;
  };
  auto count_tiles = [&](u32 s) {
    if constexpr (SHARED) {
      const i32 p0 = sh.pos0[s], n = (i32)sh.n[s];
      return n ? max(1u, seen_tiles<16>(a, p0, last_pos(s, p0, n), first_key(s)).n) + GAP : 0u;
    } else {
      const SeqView v = seq_view(a, s);
      const u32 n = short_unit_count(a, v);
      sh.pos0[s] = v.pos0; sh.n[s] = n ? (unsigned char)v.n : (unsigned char)0;
      return n;
    }
  };
  // Pairs dealt out whole: `cap` tiles of one at most to a workgroup, as few as there are workgroups for, but 32, and more (up to 64)
  // where results would be more than groups of groups take (65531 keys in 4 bits: 21.9 us with 64 results a pair, 23.2 with 128; 16384
  // keys: 19.3 with 16, 16.5 with 32). Then `pre` counts workgroups, else units.
  const u32 pairs = n_views(a) * a.nkv;
  u32 U, cap;
  bool whole;
  auto choose = [&](u32 units, u32 of) {             // (of = nwg - pairs: these are always enough)
    cap = pairs <= nwg / 2 ? max(max(32u, (units + of - 1) / of), min(64u, units / (pairs * (SHORT_GROUP * SHORT_GROUP)))) : ~0u;
    whole = cap <= 64;
  };
  if (n_views(a) <= 64) {                                 // every wave for itself, all the same: nobody waits
    const u32 n = lane < n_views(a) ? count_tiles(lane) : 0u;
    u32 sum = wave_sums(n * a.nkv);
    const u32 units = U = (u32)__builtin_amdgcn_readlane((i32)sum, 63);
#pragma unroll 1
    for (u32 of = nwg;; of = nwg - pairs) {
      choose(units, of);
      if (!whole) break;
      const u32 x = wave_sums((SHARED && n ? n - GAP + cap - 1 : n + cap - 1) / cap * a.nkv), wgs = (u32)__builtin_amdgcn_readlane((i32)x, 63);
      if (wgs <= nwg) { sum = x; U = wgs; break; }
    }
    if (lane < n_views(a)) sh.pre[lane + 1] = sum;
    if (lane == 0) sh.pre[0] = 0;
    __builtin_amdgcn_wave_barrier();
  } else {
    prefix_sums<NW>(sh.pre, sh.wave_sum, n_views(a), [&](u32 s) { return count_tiles(s) * a.nkv; });
    choose(scalar(sh.pre[n_views(a)]), nwg - pairs);
    if (whole) {
      __syncthreads();
      prefix_sums<NW>(sh.pre, sh.wave_sum, n_views(a), [&](u32 s) {
        const i32 p0 = sh.pos0[s], n = (i32)sh.n[s];
        return n ? (max(1u, seen_tiles<16>(a, p0, last_pos(s, p0, n), first_key(s)).n) + cap - 1) / cap * a.nkv : 0u;
      });
    }
    U = scalar(sh.pre[n_views(a)]);
  }
  const u32 wg_units = max(1u, (U + nwg * NW - 1) / (nwg * NW)) * NW;
  if (whole ? wg >= U : wg * wg_units >= U) return;
  if (threadIdx.x < 2) sh.last[threadIdx.x] = sh.need[threadIdx.x] = 0;
  typedef const __attribute__((address_space(4))) u32 const_u32;
  // a pair of a sequence and a kv head: its first unit and number of tiles, its rows, and which tiles those are
  struct Pair { u32 s, g, first, nv, t0, n, row, zb, wlo; i32 pos0; };
  auto last_of = [&](const Pair& p) { return p.pos0 + (SHARED && p.s >= a.n_seqs ? 1 : (i32)p.n) - 1; };      // position of the last query
  auto pair_of = [&](u32 s, u32 g) {
    Pair p;
    p.s = s; p.g = g;
    u32 of = s;                                      // the sequence whose table and first token it has
    if constexpr (SHARED) { if (s >= a.n_seqs) of = scalar(sh.link[s]); }
    p.t0 = (u32)max(0, min((i32)((const_u32*)(u64)uniform_ptr((const u32*)a.cu))[of], (i32)a.n_tokens));
    p.n = scalar(sh.n[s]); p.pos0 = (i32)scalar((u32)sh.pos0[s]);
    const Seen e = seen_tiles<16>(a, p.pos0, last_of(p), SHARED ? scalar(first_key(s)) : 0u);
    p.zb = scalar(e.zb); p.wlo = scalar(e.wlo); p.nv = scalar(max(1u, e.n));
    p.first = whole ? 0u : scalar(sh.pre[s]) + g * (p.nv + GAP) + GAP;
    p.row = a.table_row ? scalar(a.table_row[of]) : of;
    return p;
  };
  auto pair_at = [&](u32 u) {                        // (whole pairs: u = the workgroup)
    const u32 s = scalar(last_at_most(sh.pre, n_views(a), u)), in = u - scalar(sh.pre[s]);
    return pair_of(s, in / (scalar(sh.pre[s + 1] - sh.pre[s]) / a.nkv));
  };
  auto pair_after = [&](const Pair& p) {             // (there is one)
    if (p.g + 1 < a.nkv) { Pair q = p; ++q.g; q.first += q.nv + GAP; return q; }
    u32 s = p.s + 1;
    while (scalar(sh.pre[s + 1]) == scalar(sh.pre[s])) ++s;
    return pair_of(s, 0);
  };
  // the workgroup's run, and this wave's share of it
  Pair cur = pair_at(whole ? wg : wg * wg_units);
  u32 wg0 = wg * wg_units, wg1 = min(wg0 + wg_units, U), from = 0;         // from: the first workgroup of the pair (whole pairs)
  if (whole) {
    const u32 per = (cur.nv + cap - 1) / cap;
    from = scalar(sh.pre[cur.s]) + cur.g * per;
    wg0 = cur.nv * (wg - from) / per; wg1 = cur.nv * (wg - from + 1) / per;
  }
  const u32 quantum = (wg1 - wg0 + NW - 1) / NW, u0 = min(wg0 + w * quantum, wg1), u1 = min(u0 + quantum, wg1);
  auto first_wg = [&](const Pair& p) { return whole ? from : p.first / wg_units; };
  auto n_wgs = [&](const Pair& p) { return whole ? (p.nv + cap - 1) / cap : (p.first + p.nv - 1) / wg_units - p.first / wg_units + 1; };
  const TileLane at = Tile::lane_offsets();
  typename Tile::Query q[CT];
  i32 qpos[CT];                                      // position of the lane's row (no row: before every key)
  auto load_q = [&](const Pair& p) {
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      const u32 r = c * 16 + lc, rr = min(r, p.n * a.G - 1), tok = rr / a.G, h = rr - tok * a.G;
      qpos[c] = r < p.n * a.G ? (SHARED && p.s >= a.n_seqs ? p.pos0 : p.pos0 + (i32)tok) : -1;
      Tile::load_query(a.q + (u64)(p.t0 + tok) * a.qs + (u64)(p.g * a.G + h) * HD, q[c]);
    }
  };
  ShortAcc<HD, BITS> acc[CT];
  auto clear = [&]() {
#pragma unroll
    for (int c = 0; c < CT; ++c) acc[c].init();
  };
  auto finish = [&](const Pair& p) {
    if constexpr (SHARED) {
      if (is_joined(a, sh, p.s)) {
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          const float l = quad_sum(acc[c].l);
          const u32 r = c * 16 + lc, tok = r / a.G;
          if (r >= p.n * a.G) continue;
          float* const x = row_result<HD>(p.s < a.n_seqs ? 1u : 0u, p.row, p.t0, tok, p.g * a.G + r - tok * a.G);
          if (lg == 0) *(float2*)x = make_float2(acc[c].m, l);
          if constexpr (BITS == 16) {
#pragma unroll
            for (int d = 0; d < HD / 16; ++d) *(floatx4_t*)(x + 4 + d * 16 + lg * 4) = acc[c].o[d];
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int d = 0; d < HD / 16; d += 4) *(floatx4_t*)(x + 4 + Tile::o_dim(d, lg, i)) = floatx4_t{acc[c].o[d][i], acc[c].o[d + 1][i], acc[c].o[d + 2][i], acc[c].o[d + 3][i]};
          }
        }
        return;
      }
    }
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      const float l = quad_sum(acc[c].l), inv = l == 0.f ? 0.f : 1.0f / l;
      const u32 r = c * 16 + lc, tok = r / a.G, k = (p.g * a.G + r - tok * a.G) * HD;
      if (r >= p.n * a.G) continue;
      if constexpr (BITS == 16) {
#pragma unroll
        for (int d = 0; d < HD / 16; ++d)
          *(uint2*)out_at(a, p.t0 + tok, k + d * 16 + lg * 4) =
              make_uint2(half_pair(acc[c].o[d][0] * inv, acc[c].o[d][1] * inv), half_pair(acc[c].o[d][2] * inv, acc[c].o[d][3] * inv));
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int d = 0; d < HD / 16; d += 4)
            *(uint2*)out_at(a, p.t0 + tok, k + Tile::o_dim(d, lg, i)) =
                make_uint2(half_pair(acc[c].o[d][i] * inv, acc[c].o[d + 1][i] * inv), half_pair(acc[c].o[d + 2][i] * inv, acc[c].o[d + 3][i] * inv));
      }
    }
  };
  auto key_of = [&](const Pair& p, u32 u) { const u32 l = u - p.first; return (l < p.zb ? l : p.wlo + l - p.zb) * 16; };    // first key of the unit's tile
  auto block_of = [&](const Pair& p, u32 key) {      // (a pair without keys has no block either)
    return p.pos0 + (i32)p.n > 0 ? ((const_u32*)(u64)uniform_ptr(a.tables + (u64)p.row * a.max_blocks))[key / 16] : ~0u;
  };
  auto edge_of = [&](const Pair& p, u32 key, bool in_cache) {      // some row does not see the whole tile
    const i32 k = (i32)key, p1 = last_of(p);
    return !(k + 15 <= p.pos0 && in_cache && (!a.window || k > p1 - (i32)a.window || key + 16 <= a.sinks));
  };
  auto see = [&](u32 key, bool in_cache, u32 (&vis)[CT]) {
#pragma unroll
    for (int c = 0; c < CT; ++c) vis[c] = in_cache ? sees(a, qpos[c], (i32)(key + lg * 4)) : 0u;
  };
  clear();
  if (SHARED && !whole && u0 < u1 && u0 != wg0) cur = pair_at(u0);
  if (u0 < u1 && (!SHARED || cur.first < u1)) {
    if (!SHARED && u0 != wg0 && !whole) cur = pair_at(u0);
    // the tile to ask for next: its unit, pair and block id (asked for a tile ahead)
    Pair ap = cur;
    u32 au = SHARED ? max(u0, cur.first) : u0, ak = key_of(ap, au), aid = block_of(ap, ak);
    Tile tile[NT];
    u32 k0[NT];
    bool in_cache[NT], strange = false;
    auto ask = [&](int j) {                          // into slot j, unless the run has been asked for
      if (au >= u1) return;
      k0[j] = ak;
      in_cache[j] = aid < a.n_blocks;
      tile[j].load(a, at, min(aid, a.n_blocks - 1), ap.g);
      if (++au < u1) {
        if (au == ap.first + ap.nv) {
          ap = pair_after(ap);
          if constexpr (SHARED) { au = ap.first; if (au >= u1) return; }
        }
        ak = key_of(ap, au);
        aid = block_of(ap, ak);
      }
    };
    load_q(cur);
#pragma unroll
    for (int j = 0; j < NT; ++j) ask(j);
    u32 u = SHARED ? max(u0, cur.first) : u0;
    auto step = [&](int j) {                         // the tile of slot j; whether its pair, or the run, ends with it
      if (cur.pos0 + (i32)cur.n > 0) {
        const bool edge = edge_of(cur, k0[j], in_cache[j]);
        u32 vis[CT] = {};
        if (edge) {
          see(k0[j], in_cache[j], vis);
          u32 any = 0;
#pragma unroll
          for (int c = 0; c < CT; ++c) any |= vis[c];
          strange |= tile[j].take_strange_out(any);
        }
#pragma unroll
        for (int c = 0; c < CT; ++c)
          if (!SHARED || !c || c * 16u < cur.n * a.G) acc[c].add(tile[j], q[c], a.c, edge, vis[c]);
      }
      ask(j);
      ++u;
      return u == u1 || u == cur.first + cur.nv;
    };
    for (u32 j = 0;;) {
      bool ends;
      switch (j) {
        case 0: ends = step(0); j = 1; if (ends) break; [[fallthrough]];
        case 1: ends = step(1); j = 2 % NT; if (ends || NT == 2) break; [[fallthrough]];
        case 2: ends = step(2 % NT); j = 3 % NT; if (ends || NT == 3) break; [[fallthrough]];
        default: ends = step(3 % NT); j = 0;
      }
      if (!ends) continue;
      if (strange) {                                 // (an edge tile had values that are not finite: they go to the rows that see them)
        for (u32 x = max(u0, cur.first); x < u; ++x) {
          const u32 key = key_of(cur, x), b = block_of(cur, key);
          if (!edge_of(cur, key, b < a.n_blocks)) continue;
          Tile t;
          t.load(a, at, min(b, a.n_blocks - 1), cur.g);
          u32 vis[CT];
          see(key, b < a.n_blocks, vis);
#pragma unroll
          for (int c = 0; c < CT; ++c) give_strange<HD, BITS>(t, acc[c].o, vis[c]);
        }
        strange = false;
        if (u < u1) {                                // (the tiles on their way are asked for again: none of them stays in registers over this)
          ap = u == cur.first + cur.nv ? pair_after(cur) : cur;
          au = SHARED ? max(u, ap.first) : u;
          ak = key_of(ap, au);
          aid = block_of(ap, ak);
#pragma unroll
          for (int x = 0; x < NT; ++x) ask(x);
          j = 0;
        }
      }
      const bool done = u == cur.first + cur.nv;
      if (done && cur.first >= u0) finish(cur);                             // the pair is this wave's alone
      else if (cur.first < u0) leave_in_lds<HD, BITS, CT, NW>(sh, w, acc);      // its beginning is another wave's
      if (u == u1) break;                                                   // (a pair that begins here and goes on: in acc)
      if constexpr (SHARED) {
        const Pair next = pair_after(cur);
        if (next.first >= u1) break;
        cur = next;
        u = cur.first;
      } else cur = pair_after(cur);
      load_q(cur);
      clear();
      wait_loads();      // (the compiler does not know any more which slot's loads are the oldest: it would wait for all of them at every turn)
    }
  }
  // The rest is a workgroup's end, once per launch.
  const bool goes_on = u0 < u1 && cur.first >= u0 && u1 < cur.first + cur.nv && (!SHARED || cur.first < u1);
  if (goes_on && (whole || cur.first + cur.nv > wg1)) leave_in_lds<HD, BITS, CT, NW>(sh, NW, acc);
  __syncthreads();
  // pairs that other workgroups share, all waves at each: the one that the run begins inside of (0), the one that begins in it (1)
  const u32 group = wg / SHORT_GROUP, group0 = group * SHORT_GROUP;
  u32 *const pair_ctr = a.ctr + 2, *const group_ctr = pair_ctr + nwg;        // (pairs by their first workgroup)
  // a pair's results and those of its groups: which of a workgroup's (group's) two slots, by whether the pair begins before it
  auto piece = [&](u32 x, u32 first) { return a.part + (u64)(2 * x + (x == first ? 1u : 0u)) * short_slot<HD, CT>(); };
  auto group_piece = [&](u32 x, u32 first) { return a.part + (u64)(2 * (nwg + x) + (x == first / SHORT_GROUP ? 1u : 0u)) * short_slot<HD, CT>(); };
  ShortMerge<HD, BITS, CT, NW> all;
  auto finish_all = [&](const Pair& p) {
    if constexpr (SHARED) {
      if (is_joined(a, sh, p.s)) {
        const float sum = quad_sum(all.l);
        if (!all.live) return;
        const u32 r = all.c * 16 + lc, tok = r / a.G;
        float* const x = row_result<HD>(p.s < a.n_seqs ? 1u : 0u, p.row, p.t0, tok, p.g * a.G + r - tok * a.G);
        if (all.d0 == 0 && lg == 0) *(float2*)x = make_float2(all.m, sum);
        if constexpr (BITS == 16) {
#pragma unroll
          for (int t = 0; t < all.T; ++t) *(floatx4_t*)(x + 4 + (all.d0 + t) * 16 + lg * 4) = all.o[t];
        } else {
#pragma unroll
          for (int t = 0; t < all.T; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[4 + Tile::o_dim((int)all.d0 + t, lg, i)] = all.o[t][i];
        }
        return;
      }
    }
    const float l = quad_sum(all.l), inv = l == 0.f ? 0.f : 1.0f / l;
    const u32 r = all.c * 16 + lc, tok = r / a.G, k = (p.g * a.G + r - tok * a.G) * HD;
    if (!all.live) return;
    if constexpr (BITS == 16) {
#pragma unroll
      for (int t = 0; t < all.T; ++t)
        *(uint2*)out_at(a, p.t0 + tok, k + (all.d0 + t) * 16 + lg * 4) =
            make_uint2(half_pair(all.o[t][0] * inv, all.o[t][1] * inv), half_pair(all.o[t][2] * inv, all.o[t][3] * inv));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f16_t* const x = out_at(a, p.t0 + tok, k + Tile::o_dim((int)all.d0, lg, i));
        const u32 pair = half_pair(all.o[0][i] * inv, all.o[all.T - 1][i] * inv);
        if constexpr (all.T == 2) *(u32*)x = pair; else *x = (f16_t)pair;
      }
    }
  };
#pragma unroll 1
  for (u32 which = 0; which < 2; ++which) {
    const Pair p = pair_at(whole ? wg : which ? wg1 - 1 : wg0);
    const u32 end = p.first + p.nv, f = first_wg(p), np = n_wgs(p);
    if (which ? p.first < wg0 || end <= (whole ? quantum : wg1) : p.first >= wg0) continue;      // (a pair in one run: its wave has finished it)
    if (SHARED && !whole && which && p.first >= wg1) continue;           // (it begins behind the run)
    const u32 x0 = which ? (p.first - wg0) / quantum : 0u, x1 = (min(end, wg1) - wg0 + quantum - 1) / quantum;
    all.sum(x0, x1, p.n * a.G, [&](u32 x) { return LdsResult<Shared>{sh, which && x == x0 ? (u32)NW : x}; });
    if (np == 1) { finish_all(p); continue; }
    all.leave(a.part + (u64)(2 * wg + which) * short_slot<HD, CT>());
    if (threadIdx.x == 0) {
      const bool grouped = np > SHORT_GROUP;
      sh.ctr[which] = grouped ? group_ctr + 2 * group + (f >= group0 ? 1u : 0u) : pair_ctr + f;
      sh.need[which] = grouped ? min(f + np, group0 + SHORT_GROUP) - max(f, group0) : np;
    }
  }
  if (goes_on && !whole && cur.first + cur.nv <= wg1) {
#pragma unroll 1
    for (u32 x = w + 1; x < NW && wg0 + x * quantum < cur.first + cur.nv; ++x) add_from_lds<HD, BITS, CT, NW>(sh, x, acc);
    finish(cur);
  }
  // counts one result more, of lane i for pair i, when all waves' are in memory; whether it was the last one
  auto count = [&](bool mine, u32* ctr, u32 n) {
    if (!mine) return;
    const bool last = __hip_atomic_fetch_add(ctr, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == n - 1;
    if (last) __hip_atomic_store(ctr, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    sh.last[lane] = last;
  };
  asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
  __syncthreads();
  if (threadIdx.x < 2) count(sh.need[lane] != 0, sh.ctr[lane], sh.need[lane]);
  __syncthreads();
#pragma unroll 1
  for (u32 which = 0; which < 2; ++which) {
    if (!scalar(sh.last[which])) continue;
    const Pair p = pair_at(whole ? wg : which ? wg1 - 1 : wg0);
    const u32 f = first_wg(p), np = n_wgs(p), rows = p.n * a.G;
    auto of_wg = [&](u32 x) { return FarResult<HD>{piece(x, f)}; };
    if (np > SHORT_GROUP) {                          // this workgroup's group, then, if it is the last of them, the groups
      all.sum(max(f, group0), min(f + np, group0 + SHORT_GROUP), rows, of_wg);
      all.leave(group_piece(group, f));
      asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
      __syncthreads();
      if (threadIdx.x < 2) count(lane == which, pair_ctr + f, (f + np - 1) / SHORT_GROUP - f / SHORT_GROUP + 1);
      __syncthreads();
      if (!scalar(sh.last[which])) continue;
      all.sum(f / SHORT_GROUP, (f + np - 1) / SHORT_GROUP + 1, rows, [&](u32 x) { return FarResult<HD>{group_piece(x, f)}; });
    } else all.sum(f, f + np, rows, of_wg);
    finish_all(p);
  }
}

// ---- many rows: prompts and their chunks -------------------------------------------------------------------------------------
// One workgroup (eight waves of CT tiles of 16 rows) per (sequence, kv head, 128 CT rows): keys and values come once per workgroup, 64
// keys a step, into a ring in LDS that every wave reads its operands from (order in LDS: attn_prompt). Halves are fetched straight
// into the ring, keys by waves 0-3 and values by waves 4-7, three and two steps ahead. 4-bit tiles come into registers a step ahead,
// and the same waves turn keys and values into halves in that same order, so that a value is converted once per workgroup.
// Waves 4-7 are half a step behind waves 0-3 (a barrier more at the start, one less at the end): of the two waves of a SIMD one has
// its products, those of the last step's probabilities with the values and this step's scores, while the other one has its
// softmax. Operands come PROMPT_PIPE - 1 groups ahead. What stands between is kept short: a step's 40 scalar instructions for
// block ids, bounds and addresses cost a tenth of the time when they were 120, and block ids on their way (scalar loads, the
// same counter as LDS) make every wait for an operand one for them.
// The keys of a step: those of the sinks, then from the first one that the item's first query sees to the last one of its last; a
// wave skips the steps that none of its own rows see. Items come from a counter, the last queries first, each asked for an item
// ahead. With fewer items than workgroups the keys of each are cut into parts, whose results a second kernel adds up.
// Bound by the instructions of the softmax (32 exponentials and 87 others a lane and step) and the products in turn: 2048 queries at
// 16384 keys in 4 bits (32 q, 8 kv heads of 128) 547 us, 0.94 PFLOP/s, where the library's largest products reach 1.08; two prompts of 4000
// behind a window of 1024 168 us, 0.70 PFLOP/s: an item is 17 steps, and its start (queries, ids, the first tiles) and end another 3.
#define PROMPT_PIPE 3             // groups of operands on their way from LDS and in use
#define PROMPT_RING (128u * 1024u)
#define PROMPT_SLOT(HD) (PROMPT_ROWS * ((HD) + 2u))      // floats of a part's result: maximum and sum of every row, then its output
template <typename View>
struct PromptRoom {
  alignas(256) unsigned char ring[PROMPT_RING];
  u32 pre[PAGED_MAX_SEQS + 1], wave_sum[PAGED_WAVES];
  // the item after this one, and whether some step of it had values that are not finite: by the item's number among the workgroup's, so that no
  // wave has to wait at its end for those that read them
  u32 next_item[2], strange[3];
  View view[PAGED_MAX_SEQS];         // (an item begins without asking memory for them: two prompts of 4000 behind a window, four items a workgroup: 169 us -> 165)
};
typedef PromptRoom<SeqView> PromptShared;
struct SharedRoom : PromptRoom<SharedView> { u32 flat[PAGED_MAX_SEQS + 1], sum[2]; };      // units of the groups before each; of the few rows' tiles, of prompt items' steps
template <typename A> using PromptRoomOf = typename std::conditional<is_shared<A>, SharedRoom, PromptShared>::type;
template <typename A, typename F>
__device__ __forceinline__ PromptItem prompt_item(const A& a, const u32* pre, u32 item, F view) {
  PromptItem it;
  const u32 gi = pre[a.n_seqs] - 1 - item / a.nkv;             // the last queries (the longest walks) first
  it.g = item % a.nkv;
  it.s = last_at_most(pre, a.n_seqs, gi);
  const auto v = view(it.s);
  it.r0 = (gi - pre[it.s]) * PROMPT_ROWS;
  it.rows = min(PROMPT_ROWS, v.n * a.G - it.r0);
  it.t0 = v.t0;
  it.p0 = v.pos0 + (i32)(it.r0 / a.G);
  it.p1 = v.pos0 + (i32)((it.r0 + it.rows - 1) / a.G);
  it.lo = v.lo();
  it.row = it.s;
  return it;
}

// Values of one block that are not finite, given to the rows that see them (vis: bits of the lane's four keys 4 (lane / 16) ..).
template <int HD, int BITS, int CT>
__device__ __forceinline__ void give_strange_block(const PagedArgs& a, u32 id, u32 g, const u32 (&vis)[CT], floatx4_t (&o)[CT][HD / 16]) {
  const TileLane at = CacheTile<HD, BITS>::lane_offsets();
  CacheTile<HD, BITS> t;
  t.load(a, at, id, g);
  if constexpr (BITS == 16) {
#pragma unroll
    for (int c = 0; c < CT; ++c) give_strange<HD, 16>(t, o[c], vis[c]);
  } else {
    // a scale of 255 makes 32 dimensions of a key's value NaN: which of its scales, and for whom
    global_byte* const sc = uniform_global((const unsigned char*)a.cache + ((u64)id * a.nkv + g) * (17 * HD)) + opaque((threadIdx.x & 63) >> 4) * 4 + 16 * HD + HD / 2;
#pragma unroll
    for (int k = 0; k < HD / 32; ++k) {
      u32 odd = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) odd |= (sc[k * 16 + i] == 255 ? 1u : 0u) << i;
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const float nan = quad_max(odd & vis[c] ? 1.f : 0.f) > 0.f ? __uint_as_float(0x7FC00000u) : 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) { o[c][2 * k][i] += nan; o[c][2 * k + 1][i] += nan; }
      }
    }
  }
}

// (nothing is moved over either: the products belong on one side)
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
  __builtin_amdgcn_sched_barrier(0);
}
template <int N> __device__ __forceinline__ void wait_dma() { asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory"); }
__device__ __forceinline__ float* own_parts(const PagedArgs& a) { return a.prompt_part; }
__device__ __forceinline__ float* own_parts(const SharedArgs& a) { return a.own_part; }
// FLAT: the groups' shared keys in place of prompts, workgroup wg's run of them. All rows see all keys, so what is done for masks falls away, but
// for blocks outside the cache. cut_for: workgroups that few items' keys are cut into parts for, where those are not all (nwg)
template <int HD, int BITS, bool FLAT = false, typename A>
__device__ __forceinline__ void paged_prompt(const A& a, PromptRoomOf<A>& sh, u32 wg, u32 nwg, bool behind_short, FlatRun run = FlatRun{0, 0}, u32 cut_for = 0) {
  constexpr bool SHARED = is_shared<A>;
  constexpr int CT = PROMPT_CT;
  constexpr u32 BLK = 16 * HD * 2, NB = 4, STAGE = 2 * NB * BLK, NS = BITS == 4 ? 2 : (PROMPT_RING / STAGE > 6 ? 6 : PROMPT_RING / STAGE), TPW = BLK / 1024;
  const u32 lane = threadIdx.x & 63, w = (u32)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lg = lane >> 4, lc = lane & 15;
  if constexpr (!SHARED)                             // (else they are there)
    prefix_sums<PAGED_WAVES>(sh.pre, sh.wave_sum, a.n_seqs, [&](u32 s) {
      sh.view[s] = seq_view(a, s);
      return prompt_items(a, sh.view[s]);
    });
  const u32 items = FLAT ? 0u : (u32)__builtin_amdgcn_readfirstlane(sh.pre[a.n_seqs]) * a.nkv, parts = FLAT ? 1u : prompt_parts(a, items, cut_for ? cut_for : nwg), total = FLAT ? run.end : items * parts;
  u32* const ctr = a.ctr;
  const u32 lds0 = (u32)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)sh.ring;
  // fetching halves: waves 0-3 the K of a block each, waves 4-7 the V (places in LDS: attn_prompt)
  const bool fk = w < 4;
  const u32 ahead = fk ? NS - 1 : NS - 2;          // stages that a wave's fetches are ahead of its scores
  const u32 fb = w & 3u, f_lds = lds0 + w * BLK;
  const u32 k_tok = (lc & 4) * 2 + (lc & 3) + (((lc >> 3) ^ fb) & 1u) * 4;    // the key that lies at this lane's place of a K tile
  const u32 voff = fk ? k_tok * (HD * 2) + lg * 16 : ((lg >> 1) * 16 + lc) * 32 + (lg & 1) * 16, vstep = fk ? 64 : 1024;
  const u32 k_at[2] = {(lc >> 3) * BLK + lg * 256 + (lc >> 3) * 128 + (lc & 7) * 16, (lc >> 3) * BLK + lg * 256 + ((lc >> 3) ^ 1u) * 128 + (lc & 7) * 16};
  const u32 v_at = NB * BLK + (lg >> 1) * BLK + (lg & 1) * 256 + lc * 16;
  // A lane's places in a 4-bit record, and where its four dimensions of 8 values (tokens 8 th ..) lie in a block of the ring: it writes them in
  // an order of its own (x ^ turn4, with the bytes of `pick` and `odd`), so that 16 lanes write to all banks at a time (all in one
  // order they meet in an eighth of them: two fifths of the kernel's LDS cycles)
  const u32 vl = HD == 128 ? lane >> 1 & 15 : lc, vh = HD == 128 ? lane & 1 : 0u, th = HD == 128 ? lane >> 5 : lg & 1, turn4 = HD == 128 ? vl >> 1 & 3 : vl >> 2 & 3;
  const u32 d4 = HD == 128 ? vl * 8 + vh * 4 : vl * 4;
  const TileLane at4 = {opaque(k_tok * (HD / 2) + lg * 4), opaque((th * 32 + vl) * (HD / 8)), opaque(k_tok), opaque(vl / (HD == 128 ? 4 : 8) * 16 + th * 8)};
  const u32 to4 = opaque(d4 / 32 * 1024 + (d4 % 32 / 16 * 2 + th) * 256 + d4 % 16 * 16 + turn4 * 16);
  const u32 pick = opaque((turn4 & 2 ? 0x0C0C0001u : 0x0C0C0100u) + vh * 0x0202u), odd = opaque(turn4 & 1 ? 0x02020202u : 0u);
  typedef const __attribute__((address_space(4))) u32 const_u32;
  if (threadIdx.x < 3) sh.strange[threadIdx.x] = 0;
  __syncthreads();
  // (behind the short part a workgroup may come late: then its first item comes from the counter too)
  u32 turn = FLAT ? run.from : wg;
  if (!FLAT && behind_short && total) {
    if (threadIdx.x == 0) sh.next_item[1] = __hip_atomic_fetch_add(ctr, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    turn = (u32)__builtin_amdgcn_readfirstlane(sh.next_item[1]);
  }
  for (u32 nth = 0; turn < total; ++nth) {
    u32 after = 0, *const strange = sh.strange + nth % 3;
    if (threadIdx.x == 0) {
      if constexpr (!FLAT) after = (behind_short ? 0u : nwg) + __hip_atomic_fetch_add(ctr, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      sh.strange[(nth + 1) % 3] = 0;                            // (read last two items ago)
    }
    const u32 this_turn = turn, item = turn / parts, part = turn - item * parts;
    PromptItem it;
    FlatPiece piece;
    if constexpr (FLAT) {
      const u32 of = last_at_most(sh.flat, a.n_groups, turn);
      it = flat_piece(a, sh.view[a.n_seqs + of], of, sh.flat[of], turn, total, piece);
      if (!piece.any) return;                        // (the end of the run, within an item's lead)
    } else it = prompt_item(a, sh.pre, item, [&](u32 s) { return sh.view[s]; });
    it.s = (u32)__builtin_amdgcn_readfirstlane(it.s); it.g = (u32)__builtin_amdgcn_readfirstlane(it.g); it.r0 = (u32)__builtin_amdgcn_readfirstlane(it.r0);
    it.rows = (u32)__builtin_amdgcn_readfirstlane(it.rows); it.t0 = (u32)__builtin_amdgcn_readfirstlane(it.t0);
    it.p0 = __builtin_amdgcn_readfirstlane(it.p0); it.p1 = __builtin_amdgcn_readfirstlane(it.p1);
    if constexpr (SHARED) { it.lo = (u32)__builtin_amdgcn_readfirstlane(it.lo); it.row = (u32)__builtin_amdgcn_readfirstlane(it.row); }
    Seen e = {0, 0, 0};
    if constexpr (FLAT) e.n = (u32)(it.p1 + 1) / 64; else e = seen_tiles<64>(a, it.p0, it.p1, SHARED ? it.lo : 0u);
    const u32 zb = FLAT ? 0u : (u32)__builtin_amdgcn_readfirstlane(e.zb), wlo = FLAT ? 0u : (u32)__builtin_amdgcn_readfirstlane(e.wlo), n_steps = (u32)__builtin_amdgcn_readfirstlane(e.n);
    u32 per = (n_steps + parts - 1) / parts, s_lo = min(part * per, n_steps), s_hi = min(s_lo + per, n_steps);
    if constexpr (FLAT) { s_lo = (u32)__builtin_amdgcn_readfirstlane(piece.s_lo); s_hi = (u32)__builtin_amdgcn_readfirstlane(piece.s_hi); }
    const u32 last_block = (u32)max(0, it.p1) / 16;
    const u32 row = SHARED ? it.row : a.table_row ? (u32)__builtin_amdgcn_readfirstlane(a.table_row[it.s]) : it.s;
    const_u32* const bt = (const_u32*)(u64)uniform_ptr(a.tables + (u64)row * a.max_blocks);
    auto tile_of = [&](u32 s) { return s < zb ? s : wlo + s - zb; };          // 64 keys from 64 times this
    auto block_id = [&](u32 s, u32 b) { return bt[min(NB * tile_of(min(s, n_steps ? n_steps - 1 : 0u)) + b, last_block)]; };
    // this wave's rows
    const u32 wr = w * (16 * CT);
    const bool live = wr < it.rows;
    const i32 wp0 = FLAT ? it.p0 : it.p0 + (i32)((it.r0 % a.G + wr) / a.G), wp1 = FLAT ? it.p0 : it.p0 + (i32)((it.r0 % a.G + min(wr + 16 * CT, it.rows) - 1) / a.G);
    f16x8_t q[CT][HD / 32];
    i32 qpos[CT];                                    // position of the lane's row (no row: before every key)
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      const u32 r = wr + c * 16 + lc, rr = it.r0 + min(r, it.rows - 1), tok = rr / a.G, h = rr - tok * a.G;
      qpos[c] = r < it.rows ? it.p0 - (i32)(it.r0 / a.G) + (i32)tok : -1;
      u32 token = it.t0 + tok;
      if constexpr (FLAT) token = group_token(a, sh.view, sh.view[it.s], tok);
#pragma unroll
      for (int s = 0; s < HD / 32; ++s) q[c][s] = ld_tile(a.q + (u64)token * a.qs + (it.g * a.G + h) * HD + s * 32 + lg * 8);
    }
    floatx4_t o[CT][HD / 16];
    float m[CT], l[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      m[c] = -INFINITY; l[c] = 0.f;
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) o[c][d] = floatx4_t{0.f, 0.f, 0.f, 0.f};
    }
    // bounds on a step's first key (few scalar instructions in a step: they are in the way of the others)
    const i32 none = INT32_MIN, need_hi = live ? wp1 : -1, need_lo = a.window ? wp0 - (i32)a.window - 63 : none;
    const i32 edge_hi = wr + 16 * CT > it.rows ? none : wp0 - 63, edge_lo = a.window ? wp1 - (i32)a.window : none;
    const i32 item_hi = it.p0 - 63, item_lo = a.window ? it.p1 - (i32)a.window : none;
    auto needed = [&](u32 k0) { if constexpr (FLAT) return (int)live; return ((i32)k0 <= need_hi) & (((i32)k0 > need_lo) | (k0 < a.sinks)); };                              // by some row of this wave
    auto item_edge = [&](u32 k0, u32 bad) { if constexpr (FLAT) return (int)(bad != 0); return ((i32)k0 > item_hi) | (bad != 0) | (((i32)k0 <= item_lo) & (k0 + 64 > a.sinks)); };      // not seen as a whole by every row of the item
    auto edge_of = [&](u32 k0, u32 bad) { if constexpr (FLAT) return (int)(bad != 0); return ((i32)k0 > edge_hi) | (bad != 0) | (((i32)k0 <= edge_lo) & (k0 + 64 > a.sinks)); };        // nor by every one of this wave
    u32 id[NB], my_id = 0, bad_ahead = 0;            // ids of the stage to fetch next, and of this wave's block; which blocks of the stages in the ring are outside the cache, 4 bits each
    auto next_ids = [&](u32 s) {
      const u32 first = NB * tile_of(min(s, n_steps ? n_steps - 1 : 0u));
      my_id = bt[min(first + fb, last_block)];
      if (first + NB - 1 <= last_block) {
#pragma unroll
        for (u32 b = 0; b < NB; ++b) id[b] = bt[first + b];
      } else {
#pragma unroll
        for (u32 b = 0; b < NB; ++b) id[b] = bt[min(first + b, last_block)];
      }
    };
    auto note_bad = [&]() {                          // of the stage being fetched
      bad_ahead <<= 4;
      if (max(max(id[0], id[1]), max(id[2], id[3])) >= a.n_blocks) {
#pragma unroll
        for (u32 b = 0; b < NB; ++b) bad_ahead |= (id[b] < a.n_blocks ? 0u : 1u) << (NB - 1 - b);
      }
    };
    const unsigned char* const item_cache = (const unsigned char*)uniform_ptr((const unsigned char*)a.cache + (BITS == 16 ? ((u64)(fk ? 0u : a.n_blocks) * a.nkv + it.g) * BLK : (u64)it.g * (17 * HD)));
    const u32 block_bytes = a.nkv * (BITS == 16 ? BLK : 17 * HD);
    auto my_block = [&]() { return item_cache + (u64)min(my_id, a.n_blocks - 1) * block_bytes; };
    // stage s (past the last: that one again, not used) into its place of the ring, a piece after the other
    const unsigned char* f_src = nullptr;
    u32 f_at = 0;
    auto fetch_from = [&](u32 s) {
      f_src = my_block();
      f_at = f_lds + (s % NS) * STAGE;
      note_bad();
    };
    auto fetch_piece = [&](u32 r) { dma_tile<false>(f_at + r * 1024, f_src + r * vstep, voff); };
    // 4 bits: waves 0-3 a block's keys each, waves 4-7 its values, by way of registers
    u32 raw[8], raw_s[4];
    auto fetch4 = [&]() {
      global_byte* const rec = uniform_global(my_block());
      if (fk) {
#pragma unroll
        for (u32 r = 0; r < HD / 32; ++r) {
          raw[r] = from_global<u32>(rec + at4.k + r * 16);
          raw_s[r] = *(rec + at4.ks + 16 * HD + r * 16);
        }
      } else {
        if constexpr (HD == 128) {
          const u32x4_t x = from_global<u32x4_t>(rec + at4.v + 8 * HD), y = from_global<u32x4_t>(rec + at4.v + 8 * HD + 256);
#pragma unroll
          for (int i = 0; i < 4; ++i) { raw[i] = x[i]; raw[4 + i] = y[i]; }
        } else {
          const u32x2_t x = from_global<u32x2_t>(rec + at4.v + 8 * HD), y = from_global<u32x2_t>(rec + at4.v + 8 * HD + 128);
#pragma unroll
          for (int i = 0; i < 2; ++i) { raw[i] = x[i]; raw[2 + i] = y[i]; }
        }
        const u32x2_t z = from_global<u32x2_t>(rec + at4.vs + 16 * HD + HD / 2);
        raw_s[0] = z[0]; raw_s[1] = z[1];
      }
      note_bad();
    };
    auto convert4 = [&](u32 s, u32 half) {           // half of what fetch4 brought, as halves into the ring
      unsigned char* const st = sh.ring + (s % NS) * STAGE;
      if (fk) {
        unsigned char* const to = st + fb * BLK + lane * 16;
#pragma unroll
        for (u32 r = half * (HD / 64); r < (half + 1) * (HD / 64); ++r) {
          const float sc = __uint_as_float(raw_s[r] << 23);
          *(uint4*)(to + r * 1024) = make_uint4(f16x2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(raw[r], sc, 0)), f16x2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(raw[r], sc, 1)),
                                                f16x2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(raw[r], sc, 2)), f16x2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(raw[r], sc, 3)));
        }
      } else if (HD == 128 || lane < 32) {
        // a lane: 8 tokens x 4 dimensions (of heads of 128 the lower or upper 4 of 8)
        u32 pr[8];                                   // [token], a pair of dimensions
#pragma unroll
        for (u32 i = 0; i < 8; ++i) {
          const float sc = __uint_as_float((raw_s[i / 4] >> (8 * (i % 4)) & 0xFFu) << 23);
          const u32 r = HD == 128 ? raw[i] : raw[i / 2], x = __builtin_amdgcn_perm(0u, r, HD == 64 && i & 1 ? pick + 0x0202u : pick);
          pr[i] = f16x2_bits(half ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x, sc, 1) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x, sc, 0));
        }
        unsigned char* const to = st + (NB + fb) * BLK;
#pragma unroll
        for (u32 x = 0; x < 2; ++x) {
          const u32 sel = (x & 1 ? 0x07060302u : 0x05040100u) ^ odd;
          u32 v[4];
#pragma unroll
          for (u32 i = 0; i < 4; ++i) v[i] = __builtin_amdgcn_perm(pr[2 * i + 1], pr[2 * i], sel);
          *(uint4*)(to + (to4 ^ (2 * half + x) * 16)) = make_uint4(v[0], v[1], v[2], v[3]);
        }
      }
    };
    // values of a stage that are not finite: taken out (0 times one would not be 0) by the wave that brought them, where some row of the
    // item must not see them, and given to the rows that see them at the end
    auto take_strange_out = [&](u32 s, u32 bad) {
      if (fk || s >= s_hi || !item_edge(tile_of(s) * 64, bad)) return;
      unsigned char* const v = sh.ring + (s % NS) * STAGE + (NB + fb) * BLK + lane * 16;
#pragma unroll
      for (u32 r = 0; r < BLK / 1024; ++r) {
        const uint4 x = *(const uint4*)(v + r * 1024), y = make_uint4(only_finite(x.x), only_finite(x.y), only_finite(x.z), only_finite(x.w));
        if (__ballot(x.x != y.x || x.y != y.y || x.z != y.z || x.w != y.w)) {
          *(uint4*)(v + r * 1024) = y;
          *strange = 1;
        }
      }
    };
    if constexpr (BITS == 16) {
#pragma unroll 1
      for (u32 s = 0; s < ahead; ++s) {
        next_ids(s_lo + s);
        fetch_from(s_lo + s);
#pragma unroll
        for (u32 r = 0; r < TPW; ++r) fetch_piece(r);
      }
      next_ids(s_lo + ahead);
      fetch_from(s_lo + ahead);
      wait_loads();      // (left to the compiler, the wait for the queries stands in the loop and empties the ring in every step)
    } else {
      next_ids(s_lo);
      fetch4();
      convert4(s_lo, 0);
      convert4(s_lo, 1);
      take_strange_out(s_lo, bad_ahead & 15u);
      next_ids(s_lo + 1);
      fetch4();
      next_ids(s_lo + 2);
    }
    if (threadIdx.x == 0) sh.next_item[nth & 1] = after;
    lds_barrier();
    if (!fk) lds_barrier();
    floatx4_t sc[CT][NB];
    f16x8_t pb[CT][NB / 2];
    // The products of a step, in groups of two operands (2 CT products): those of the step before's probabilities with a tile of dimensions,
    // then this step's scores. The operands come PROMPT_PIPE - 1 groups ahead, in one pipe, and a piece of a fetch now and then.
    constexpr int NPV = HD / 16, PER = HD / 64, NG = NPV + (int)NB * PER;
    f16x8_t x[PROMPT_PIPE][2];
    auto ask = [&](u32 s, int i) {
      const unsigned char *const sv = sh.ring + ((s - 1) % NS) * STAGE + v_at, *const st0 = sh.ring + (s % NS) * STAGE;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (i < NPV) x[i % PROMPT_PIPE][j] = as_f16x8(*(const uint4*)(sv + 2 * j * BLK + (i >> 1) * 1024 + (i & 1) * 512));
        else x[i % PROMPT_PIPE][j] = as_f16x8(*(const uint4*)(st0 + ((i - NPV) / PER & 2) * BLK + ((i - NPV) % PER * 2 + j) * 1024 + k_at[(i - NPV) / PER & 1]));
      }
    };
    auto products = [&](u32 s, int i, bool more) {
      if (more) ask(s, i + PROMPT_PIPE - 1);
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          if (i < NPV) o[c][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[i % PROMPT_PIPE][j], pb[c][j], o[c][i], 0, 0, 0);
          else {
            floatx4_t& y = sc[c][(i - NPV) / PER];
            const int at = (i - NPV) % PER * 2 + j;
            y = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[i % PROMPT_PIPE][j], q[c][at], at ? y : floatx4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
          }
        }
      if constexpr (BITS == 16) {
        if (i >= NPV && (i - NPV) % 2 && (i - NPV) / 2 < (int)TPW) fetch_piece((i - NPV) / 2);
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    bool scored = false;                                       // of the step before: probabilities that wait for their values
    for (u32 s = s_lo;; ++s) {
      u32 bad = 0;                                             // (asked first: a loop that begins with its products is turned around by the compiler, which then spills)
      if (s < s_hi) bad = bad_ahead >> (4 * (BITS == 16 ? ahead : 1u)) & 15u;
      if (scored) {
#pragma unroll
        for (int i = 0; i < PROMPT_PIPE - 1; ++i) ask(s, i);
#pragma unroll
        for (int i = 0; i < NPV; ++i) products(s, i, true);
      } else {
#pragma unroll
        for (int i = 0; i < PROMPT_PIPE - 1; ++i) ask(s, NPV + i);
      }
      if (s == s_hi) break;
      const u32 k0 = tile_of(s) * 64;
      const bool scores = needed(k0);
      if (scores) {
#pragma unroll
        for (int i = NPV; i < NG; ++i) products(s, i, i + PROMPT_PIPE - 1 < NG);
      } else if constexpr (BITS == 16) {
#pragma unroll
        for (u32 r = 0; r < TPW; ++r) fetch_piece(r);
      }
      scored = scores;
      if constexpr (BITS == 16) {
        if (!fk) {
          wait_dma<(int)((NS - 2) * TPW)>();                     // this wave's values of the step
          take_strange_out(s, bad);
        }
      }
      lds_barrier();
      if constexpr (BITS == 4) {                               // (behind the softmax, the barrier waits for these writes: 566 us and not 549)
        convert4(s + 1, 0);
        convert4(s + 1, 1);
        take_strange_out(s + 1, bad_ahead & 15u);
        fetch4();
      }
      // (asked for here: with them on their way a wait for an operand from LDS would be one for them too)
      next_ids(s + (BITS == 16 ? ahead + 1 : 3u));
      if (scored) {
        const bool edge = edge_of(k0, bad);
        if (edge) {
          asm volatile("" ::: "memory");                         // (a branch: few steps are)
#pragma unroll
          for (int c = 0; c < CT; ++c) {
            u32 vis = 0;                                         // bit 8 h + i: this lane's row sees its key i of the step's pair of blocks h
#pragma unroll
            for (u32 h = 0; h < NB / 2; ++h)
              if (!(bad >> (NB - 1 - (2 * h + (lg >> 1))) & 1u)) vis |= (FLAT ? 0xFFu : sees(a, qpos[c], (i32)(k0 + h * 32 + lg * 8))) << (8 * h);
#pragma unroll
            for (u32 b = 0; b < NB; ++b)
#pragma unroll
              for (int i = 0; i < 4; ++i) sc[c][b][i] = vis >> (b * 4 + i) & 1u ? sc[c][b][i] : -INFINITY;
          }
        }
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          float top = -INFINITY;
#pragma unroll
          for (u32 b = 0; b < NB; ++b) top = fmaxf(top, fmaxf(fmaxf(sc[c][b][0], sc[c][b][1]), fmaxf(sc[c][b][2], sc[c][b][3])));
          top *= a.c;
          if (__ballot(top > m[c] + 8.f)) {
            top = quad_max(top);
            const float mn = fmaxf(m[c], top);
            const float f = mn == m[c] || m[c] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[c] - mn);
            l[c] *= f;
#pragma unroll
            for (int d = 0; d < HD / 16; ++d) o[c][d] *= f;
            m[c] = mn;
          }
          const float nm = m[c] == -INFINITY ? 0.f : -m[c];
          float ps = 0.f;
#pragma unroll
          for (u32 b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[c][b][i], a.c, nm));
              ps += p;
              pb[c][b / 2][(b & 1) * 4 + i] = (_Float16)p;
            }
          l[c] += ps;
        }
      }
      if constexpr (BITS == 16) {
        fetch_from(s + 1 + ahead);
        if (fk) wait_dma<(int)((NS - 2) * TPW)>();               // this wave's keys of the next step
      }
      lds_barrier();
    }
    if constexpr (BITS == 16) wait_dma<0>();                   // (no fetch of this item is on its way any more)
    if (fk) lds_barrier();
    lds_barrier();
    if constexpr (FLAT) turn = (u32)__builtin_amdgcn_readfirstlane(piece.next);
    else turn = (u32)__builtin_amdgcn_readfirstlane(sh.next_item[nth & 1]);
    if ((u32)__builtin_amdgcn_readfirstlane(*strange)) {
#pragma unroll 1
      for (u32 s = s_lo; s < s_hi; ++s) {
        const u32 k0 = tile_of(s) * 64;
        if (!needed(k0)) continue;
        u32 bad = 0;
        for (u32 b = 0; b < NB; ++b) bad = bad << 1 | (block_id(s, b) < a.n_blocks ? 0u : 1u);
        if (!item_edge(k0, bad)) continue;
#pragma unroll 1
        for (u32 b = 0; b < NB; ++b) {
          if (bad >> (NB - 1 - b) & 1u) continue;
          u32 vis[CT];
#pragma unroll
          for (int c = 0; c < CT; ++c) vis[c] = FLAT ? 15u : sees(a, qpos[c], (i32)(k0 + b * 16 + lg * 4)) & 15u;
          give_strange_block<HD, BITS, CT>(a, block_id(s, b), it.g, vis, o);
        }
      }
      wait_loads();
    }
    // (where a row goes is worked out here: the compiler must not keep it through the loop)
    const u32 at_end = opaque(lane), lc_end = at_end & 15, lg_end = at_end >> 4;
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      const float sum = quad_sum(l[c]);
      const u32 r = wr + c * 16 + lc_end;
      if (r >= it.rows) continue;
      bool to_row = false;
      if constexpr (SHARED) to_row = FLAT ? piece.whole : parts == 1 && it.lo;
      if (to_row) {
        if constexpr (SHARED) {
          const u32 rr = it.r0 + r, tok = rr / a.G;
          float* const x = row_result<HD>(FLAT ? 0u : 1u, it.row, it.t0, tok, it.g * a.G + rr - tok * a.G);
          if (lg_end == 0) *(float2*)x = make_float2(m[c], sum);
#pragma unroll
          for (int d = 0; d < HD / 16; ++d) *(floatx4_t*)(x + 4 + d * 16 + lg_end * 4) = o[c][d];
        }
      } else if (!FLAT && parts == 1) {
        const float inv = sum == 0.f ? 0.f : 1.0f / sum;
        const u32 rr = it.r0 + r, tok = rr / a.G, k = (it.g * a.G + rr - tok * a.G) * HD + lg_end * 4;
        f16_t* const to = out_at(a, it.t0 + tok, k);
        const u32 step = a.out_tbs ? (u32)(packed_off(0, 32, a.out_tbs) - packed_off(0, 0, a.out_tbs)) : 32u, half = a.out_tbs ? 256u : 16u;      // 32 and 16 dimensions on
#pragma unroll
        for (int d = 0; d < HD / 16; ++d)
          *(uint2*)(to + (u64)(d / 2) * step + d % 2 * half) = make_uint2(half_pair(o[c][d][0] * inv, o[c][d][1] * inv), half_pair(o[c][d][2] * inv, o[c][d][3] * inv));
      } else {
        float* const slot = (SHARED && !FLAT ? own_parts(a) : a.prompt_part) + (u64)(FLAT ? flat_slot(wg, piece.begins) : this_turn) * PROMPT_SLOT(HD);
        if (lg_end == 0) *(float2*)(slot + 2 * r) = make_float2(m[c], sum);
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) *(floatx4_t*)(slot + 2 * PROMPT_ROWS + r * HD + d * 16 + lg_end * 4) = o[c][d];
      }
    }
  }
  // the last workgroup out leaves the counters as it found them
  if (!FLAT && total && threadIdx.x == 0 && __hip_atomic_fetch_add(ctr + 1, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == nwg - 1) {
    __hip_atomic_store(ctr, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(ctr + 1, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

// The parts of the prompt items added up: a wave per row, its lanes along the dimensions. `nwg_prompt`: workgroups of the launch before.
struct PromptMergeShared { u32 pre[PAGED_MAX_SEQS + 1], wave_sum[PAGED_WAVES]; };
template <int HD>
__device__ __forceinline__ void prompt_merge(const PagedArgs& a, PromptMergeShared& sh, u32 wg, u32 nwg, u32 nwg_prompt) {
  prefix_sums<PAGED_WAVES>(sh.pre, sh.wave_sum, a.n_seqs, [&](u32 s) { return prompt_items(a, seq_view(a, s)); });
  const u32 items = sh.pre[a.n_seqs] * a.nkv, parts = prompt_parts(a, items, nwg_prompt), lane = threadIdx.x & 63;
  if (parts < 2) return;
  for (u32 i = wg * PAGED_WAVES + (threadIdx.x >> 6); i < items * PROMPT_ROWS; i += nwg * PAGED_WAVES) {
    const u32 item = i / PROMPT_ROWS, r = i % PROMPT_ROWS;
    const PromptItem it = prompt_item(a, sh.pre, item, [&](u32 s) { return seq_view(a, s); });
    if (r >= it.rows) continue;
    const float* const base = a.prompt_part + (u64)item * parts * PROMPT_SLOT(HD);
    float M = -INFINITY, L = 0.f, O[HD / 64];
#pragma unroll
    for (int d = 0; d < HD / 64; ++d) O[d] = 0.f;
    for (u32 p = 0; p < parts; ++p) M = fmaxf(M, base[(u64)p * PROMPT_SLOT(HD) + 2 * r]);
    const float ref = M == -INFINITY ? 0.f : M;
    for (u32 p = 0; p < parts; ++p) {
      const float* const b = base + (u64)p * PROMPT_SLOT(HD);
      const float f = __builtin_amdgcn_exp2f(b[2 * r] - ref);
      L += b[2 * r + 1] * f;
#pragma unroll
      for (int d = 0; d < HD / 64; ++d) O[d] += b[2 * PROMPT_ROWS + r * HD + d * 64 + lane] * f;
    }
    const u32 rr = it.r0 + r, tok = rr / a.G, h = rr - tok * a.G;
#pragma unroll
    for (int d = 0; d < HD / 64; ++d) *out_at(a, it.t0 + tok, (it.g * a.G + h) * HD + d * 64 + lane) = (f16_t)half_pair(L == 0.f ? 0.f : O[d] / L, 0.f);
  }
}

// Batches that may hold both: every workgroup first its runs of the few rows' tiles, then prompt items from the counter.
template <int HD, int CT, typename A = PagedArgs> union PagedShared { ShortShared<HD, CT, PAGED_WAVES, is_shared<A>> s; PromptRoomOf<A> p; };
template <int HD, int BITS, int CT, int NT, typename A>
__device__ __forceinline__ void paged_both(const A& a, PagedShared<HD, CT, A>& sh, u32 wg, u32 nwg) {
  paged_short<HD, BITS, CT, NT, PAGED_WAVES>(a, sh.s, wg, nwg);
  __syncthreads();
  paged_prompt<HD, BITS>(a, sh.p, wg, nwg, true);
}
