// Log probabilities of given tokens with their ranks, the entropy and the most probable tokens, from rows of logits that are read once.
// With z = x * inverse temperature, c = inverse temperature * log2(e), y = x c - M for a number M near the largest x c, and S = sum 2^y:
// log p = ln 2 (y - log2 S), entropy = ln 2 (log2 S - sum y 2^y / S). M may be any number: it is one for a wave, of the largest logit of its first tile, and
// another one only where a later tile's is 2 above it, so that a logit costs one fused multiply-add ahead of its exponential; the difference of x c
// and M is rounded once, so M's own rounding falls out.
//
// Order: larger logits first, of equal ones the lower id; a key of 64 bits (the logit's bits turned into a whole number, then the id
// downwards) makes every place of it distinct. The kth largest of the first tiles' largest logits, one of every few lanes, is a bound: what is
// below it, or equal and in a later tile, is not among the k first. The keys of the others come together in LDS, each wave's apart; of more than LP_FEW (a
// wave adds a tile at most) the kth is searched for bit by bit, and what is below it thrown away. At last all are ranked, every
// one against every other.
//
// Bound by the logits' bytes, and for few rows by latencies, one after the other. Waves work on their own, each with its next tile on its way, and meet at a row's end only: tiles
// of a workgroup, with a barrier or two each, took twice as long (1021 rows of 151936 in 16 bits, no alternatives: 122 us, now 57, 5.4 TB/s). 256 rows of 128256
// floats take 26 us, 5.1 TB/s, without alternatives and 35 with 20 of them: a microsecond for the bound, two for the keys of the waves, three to five for a row's parts, while
// nothing is read. Loops over a wave's keys are not unrolled: with four instances (38 KB of code) instructions come from memory once each, and that took 59 us. One row of
// 32000 with 5 alternatives: 11.3 us (1 to start, 1 the bound, 4 the tile, 2 the keys, 3 the parts).
#pragma once
#include "blink_device.h"

#define LP_VALS 16u                // logits of a lane in a tile
#define LP_TILE (64u * LP_VALS)    // a wave's
#define LP_WAVES (BLK_THREADS / 64u)
#define LP_MOST 64u                // given tokens (a lane each), most probable tokens
#define LP_FEW 160u                // keys that a wave keeps from tile to tile at most (256 rows of 128256, 20 alternatives: 36 us; with 96 40, with 256, and so fewer workgroups at a time, 50)
#define LP_CAP (LP_FEW + LP_TILE + 8)      // (and zeros behind them)
#define LP_RANKED 96u              // keys of a workgroup that are ranked as they are (the 256 rows: 36 us; with 48 38, with 192 37)
// workgroups of a row, and keys of theirs that are joined (8 rows of 128256, 5 alternatives: 14.6 us in 32 parts, 13.8 in 16, 15.7 in 8; 64 rows with 64 of them: 48 us with
// 1024 keys, 34 with 512, 45 with 320, 58 with 128)
#define LP_MAX_PARTS 16u
#define LP_JOINED 512u
#define LP_PER_CU 4u               // workgroups that a call has for every compute unit, where its rows have the tiles (the 256 rows: 36 us; with 2, 3, 6: 46, 36, 48)
#define LP_LOWEST -3.4028235e38f
#define LP_LN2 0.69314718055994530942f
#define LP_CTR_BYTES 8192u         // of the workspace: a counter per row whose parts are joined

struct LogprobArgs {
  const void* x;
  u64 stride;
  u32 rows, V, given, k, parts;
  const i32* tokens;              // [row][given]
  const float* inverse;           // null: 1
  float* logprobs;
  i32* ranks;                     // null: not asked for
  float* entropy;                 // the same
  i32* top_ids;
  float* top_logprobs;
  u32* ctr;
  u32* results;                   // of the parts: lp_words(given, k) words each
};
// a part's result: m and sums, logits before each given one, then keys
__host__ __device__ __forceinline__ u32 lp_key_word(u32 given) { return (4 + given + 1) & ~1u; }
__host__ __device__ __forceinline__ u32 lp_words(u32 given, u32 k) { return lp_key_word(given) + 2 * k; }

template <bool TOP>
struct LogprobShared {
  alignas(16) u64 cand[TOP ? LP_WAVES * LP_CAP : 1];
  u64 top[LP_MOST];
  alignas(16) u32 group[TOP ? BLK_THREADS : 1];
  u32 kth, before[LP_WAVES][LP_MOST], n[LP_WAVES], last;
  float m[LP_WAVES], s[LP_WAVES], t[LP_WAVES];
};

__device__ __forceinline__ float lp_ordered(float x) { return fmaxf(x, -INFINITY); }      // NaN: as -inf
__device__ __forceinline__ u32 lp_high(float x) {
  const u32 b = __float_as_uint(lp_ordered(x) + 0.0f);                                    // (-0: as 0)
  return b ^ ((i32)b < 0 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ u64 lp_key(float x, u32 id) { return (u64)lp_high(x) << 32 | (0xFFFFFFFFu - id); }
__device__ __forceinline__ float lp_next_lower(float x) {      // (of a number, or +inf)
  const u32 b = __float_as_uint(x);
  return __uint_as_float(x > 0.f ? b - 1 : x < 0.f ? b + 1 : 0x80000001u);
}
__device__ __forceinline__ u32 lp_id(u64 key) { return 0xFFFFFFFFu - (u32)key; }
__device__ __forceinline__ float lp_value(u32 high) { return __uint_as_float(high ^ ((i32)high < 0 ? 0x80000000u : 0xFFFFFFFFu)); }
__device__ __forceinline__ u32 lp_below(u64 mask) { return __builtin_amdgcn_mbcnt_hi((u32)(mask >> 32), __builtin_amdgcn_mbcnt_lo((u32)mask, 0)); }     // bits of lower lanes
// what lanes of a wave write to LDS for one another (in order in hardware; the compiler is told)
__device__ __forceinline__ void lp_wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// A number that k keys of those the lanes have are not below, into sh.kth: the kth largest of the largest upper halves of groups of 16, 4 or 1 neighbouring
// lanes, two groups at least for each of the k; `mine`: the lane's largest, 0 if it has none.
template <typename Shared>
__device__ __forceinline__ void lp_kth(Shared& sh, u32 mine, u32 k) {
  u32 lanes = 1;
#pragma unroll 1
  while (lanes < 16 && 8 * k * lanes <= BLK_THREADS) {
    mine = max(mine, (u32)__shfl_xor((int)mine, (int)lanes));
    mine = max(mine, (u32)__shfl_xor((int)mine, (int)(2 * lanes)));
    lanes *= 4;
  }
  const u32 n = BLK_THREADS / lanes;
  if (threadIdx.x % lanes == 0) sh.group[threadIdx.x / lanes] = mine;
  if (threadIdx.x == 0) sh.kth = 0;
  __syncthreads();
  if (threadIdx.x < n) {
    mine = sh.group[threadIdx.x];
    u32 above = 0, not_below = 0;
#pragma unroll 4
    for (u32 j = 0; j < n; j += 4) {
      const uint4 x = *(const uint4*)(sh.group + j);
      above += (x.x > mine ? 1u : 0u) + (x.y > mine ? 1u : 0u) + (x.z > mine ? 1u : 0u) + (x.w > mine ? 1u : 0u);
      not_below += (x.x >= mine ? 1u : 0u) + (x.y >= mine ? 1u : 0u) + (x.z >= mine ? 1u : 0u) + (x.w >= mine ? 1u : 0u);
    }
    if (above < k && not_below >= k) sh.kth = mine;  // (the same one from every lane that finds it)
  }
  __syncthreads();
}
// Of the n <= LP_CAP keys of a wave's list those that are not below the kth, in the order they had; where more than LP_FEW have its logit or a larger
// one, the k first. The kth one's upper half.
__device__ __forceinline__ u32 lp_thin(u64* cand, u32& n, u32 k) {
  constexpr u32 R = (LP_CAP + 63) / 64;
  const u32 lane = threadIdx.x & 63;
  lp_wave_sync();
  u32 h[R];
#pragma unroll
  for (u32 r = 0; r < R; ++r) h[r] = r * 64 + lane < n ? (u32)(cand[r * 64 + lane] >> 32) : 0u;
  u32 high = 0, low = 0, with = n;
#pragma unroll 1
  for (u32 b = 1u << 31; b; b >>= 1) {
    const u32 up = high | b;
    u32 c = 0;
#pragma unroll
    for (u32 r = 0; r < R; ++r) c += (u32)__popcll(__ballot(h[r] >= up));
    if (c >= k) { high = up; with = c; }
  }
  if (with > LP_FEW) {
    u32 need = k;
#pragma unroll
    for (u32 r = 0; r < R; ++r) need -= (u32)__popcll(__ballot(h[r] > high));
#pragma unroll 1
    for (u32 b = 1u << 31; b; b >>= 1) {
      u32 c = 0;
#pragma unroll 1
      for (u32 i = lane; i - lane < n; i += 64) c += (u32)__popcll(__ballot(i < n && (u32)(cand[i] >> 32) == high && (u32)cand[i] >= (low | b)));
      if (c >= need) low |= b;
    }
  }
  const u64 least = (u64)high << 32 | low;
  u32 m = 0;
#pragma unroll 1
  for (u32 i = lane; i - lane < n; i += 64) {
    const u64 x = i < n ? cand[i] : 0;
    const u64 mask = __ballot(i < n && x >= least);
    if (i < n && x >= least) cand[m + lp_below(mask)] = x;       // (not behind what has been read)
    m += (u32)__popcll(mask);
  }
  lp_wave_sync();
  n = m;
  return high;
}

// Sums about M = m c, or, where that is not finite and m is (a row with nothing but a mask's lowest values, for one), about m: y = (x - m) c.
struct LpSums {
  float m, s, t;                                     // sum 2^y, sum y 2^y
  static __device__ __forceinline__ bool near(float M) { return fabsf(M) < INFINITY; }
  __device__ __forceinline__ void to(float m2, float c) {      // the same about another m
    if (m != -INFINITY && m2 != m) {                 // (nothing yet: sums of 0, or NaN)
      const float M = m * c, M2 = m2 * c, y = near(M) && near(M2) ? M - M2 : (m - m2) * c, f = __builtin_amdgcn_exp2f(y);
      t = f > 0.f ? f * __builtin_fmaf(y, s, t) : 0.f;         // (y may be -inf)
      s *= f;
    }
    m = m2;
  }
  __device__ __forceinline__ void add(LpSums o, float c) {
    const float m2 = fmaxf(m, o.m);
    to(m2, c); o.to(m2, c);
    s += o.s; t += o.t;
  }
};
__device__ __forceinline__ float lp_wave_max(float v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
__device__ __forceinline__ float lp_wave_sum(float v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
  return v;
}

// A tile as it lies in memory: 16 bytes a lane, then the next 64 times 16.
template <typename T>
struct LpTile {
  static constexpr u32 VEC = 16 / sizeof(T), NV = LP_VALS / VEC;
  typedef T vec_t __attribute__((ext_vector_type(VEC)));
  vec_t v[NV];
  static __device__ __forceinline__ u32 element(u32 j) { return (j / VEC * 64 + (threadIdx.x & 63)) * VEC + j % VEC; }
  __device__ __forceinline__ void load(const T* base, u32 at, u32 begin, u32 end) {
    if (at >= begin && at + LP_TILE <= end) {
#pragma unroll
      for (u32 i = 0; i < NV; ++i) v[i] = __builtin_nontemporal_load((const vec_t*)(base + at + element(i * VEC)));
    } else {                                         // elements outside [begin, end) are not read: -inf
#pragma unroll
      for (u32 i = 0; i < NV; ++i) {
        const u32 e = at + element(i * VEC);
#pragma unroll
        for (u32 j = 0; j < VEC; ++j) v[i][j] = e + j >= begin && e + j < end ? base[e + j] : (T)-INFINITY;
      }
    }
  }
  __device__ __forceinline__ float get(u32 j) const { return (float)v[j / VEC][j % VEC]; }
};

template <typename T, bool TOP>
__device__ __forceinline__ void token_logprobs(const LogprobArgs& a, LogprobShared<TOP>& sh, u32 wg) {
  typedef LpTile<T> Tile;
  constexpr u32 VEC = Tile::VEC;
  const u32 row = wg / a.parts, part = wg - row * a.parts, lane = threadIdx.x & 63, w = (u32)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // the row's elements are [shift, end) of what begins at the 16 bytes its first one lies in
  const T* const first = (const T*)a.x + (u64)row * a.stride;
  const u32 shift = (u32)((u64)first % 16 / sizeof(T)), end = shift + a.V;
  const T* const base = first - shift;
  const u32 tiles = (end + LP_TILE - 1) / LP_TILE, tile0 = (u32)((u64)tiles * part / a.parts) + w, tile1 = (u32)((u64)tiles * (part + 1) / a.parts);
  Tile ahead;
  if (tile0 < tile1) ahead.load(base, tile0 * LP_TILE, shift, end);
  const float inverse = a.inverse ? a.inverse[row] : 1.f;
  float c = inverse * 1.44269504088896340736f;
  if (!(inverse > 0.f) || !(c < INFINITY)) c = __uint_as_float(0x7FC00000u);
  i32 token = -1;                                    // the lane's given token, its logit, and how many come before it
  float given = 0.f;
  u32 before = 0;
  if (lane < a.given) {
    const i32 t = a.tokens[(u64)row * a.given + lane];
    if (t >= 0 && (u32)t < a.V) { token = t; given = lp_ordered((float)first[t]); }
  }
  const u32 token0 = (u32)__builtin_amdgcn_readfirstlane(token);
  const float given0 = __uint_as_float((u32)__builtin_amdgcn_readfirstlane((i32)__float_as_uint(given)));
  LpSums sum = {-INFINITY, 0.f, 0.f};                // (m: the wave's, sums: the lane's)
  u64* const cand = sh.cand + (TOP ? w * LP_CAP : 0);
  u32 n = 0;                                         // keys in cand
  float over = -INFINITY;                            // a bound: k logits of earlier tiles at least are not below it
  if constexpr (TOP) {
    float most = -INFINITY;
    if (tile0 < tile1) {
#pragma unroll
      for (u32 j = 0; j < LP_VALS; ++j) most = fmaxf(most, ahead.get(j));
    }
    lp_kth(sh, lp_high(most), a.k);
    over = sh.kth ? lp_value(sh.kth) : -INFINITY;
  }
#pragma unroll 1
  for (u32 tile = tile0; tile < tile1; tile += LP_WAVES) {
    const u32 at = tile * LP_TILE;
    const bool whole = at >= shift && at + LP_TILE <= end;
    float x[LP_VALS];
#pragma unroll
    for (u32 j = 0; j < LP_VALS; ++j) x[j] = ahead.get(j);
    if (tile + LP_WAVES < tile1) ahead.load(base, at + LP_WAVES * LP_TILE, shift, end);
    auto id = [&](u32 j) { return at + Tile::element(j) - shift; };
    auto valid = [&](u32 j) { return whole || id(j) < a.V; };      // (before the row: beyond 2^31)
    float most = -INFINITY;
#pragma unroll
    for (u32 j = 0; j < LP_VALS; ++j) most = fmaxf(most, x[j]);
    float M = sum.m * c;
    if (__ballot(LpSums::near(M) ? most * c > M + 2.f : most > sum.m)) {
      sum.to(fmaxf(sum.m, lp_wave_max(most)), c);
      M = sum.m * c;
    }
    float s[4] = {0.f, 0.f, 0.f, 0.f}, t[4] = {0.f, 0.f, 0.f, 0.f};      // (chains of a few sums: a row of one probable token loses little to rounding)
    auto add = [&](u32 j, float y) {
      const float e = __builtin_amdgcn_exp2f(y);
      s[j & 3] += e;
      t[j & 3] = __builtin_fmaf(fmaxf(y, LP_LOWEST), e, t[j & 3]);     // (0 times -inf is to be 0)
    };
    if (LpSums::near(M)) {
#pragma unroll
      for (u32 j = 0; j < LP_VALS; ++j) add(j, __builtin_fmaf(x[j], c, -M));
    } else {
      const float m = sum.m == -INFINITY ? 0.f : sum.m;
#pragma unroll
      for (u32 j = 0; j < LP_VALS; ++j) add(j, (x[j] - m) * c);
    }
    sum.s += (s[0] + s[1]) + (s[2] + s[3]);
    sum.t += (t[0] + t[1]) + (t[2] + t[3]);
    // Logits of the tile that come before the token tk, whose logit is y, by `count`: of those with a lower id the ones that are not below y, of the others those above it.
    // (y = -inf: all with a lower id, whatever they are; added where the token is.) Elements outside the row, -inf, are never counted.
    auto ranked = [&](u32 tk, float y, auto count, auto all) {
      const float lower = y == -INFINITY ? INFINITY : lp_next_lower(y);
      if (tk + shift < at || tk + shift >= at + LP_TILE) {
        const float bound = tk + shift < at ? y : lower;
        if (__ballot(most > bound)) count([&](u32 j) { return x[j] > bound; });
      } else {
        const i32 mine = (i32)(tk + shift - at) - (i32)Tile::element(0);       // (element(j) is that of j = 0 and a constant more)
        count([&](u32 j) { return x[j] > ((i32)(j / VEC * 64 * VEC + j % VEC) < mine ? lower : y); });
        if (y == -INFINITY) all(tk);
      }
    };
    if (a.ranks && a.given == 1) {
      ranked(token0, given0, [&](auto is) {          // (a lane's own: added up at the end)
#pragma unroll
        for (u32 j = 0; j < LP_VALS; ++j) before += is(j) ? 1u : 0u;
      }, [&](u32 n) { before += lane == 0 ? n : 0u; });
    } else if (a.ranks) {
#pragma unroll 1
      for (u32 g = 0; g < a.given; ++g) {
        const u32 tk = (u32)__builtin_amdgcn_readlane(token, (int)g);
        const float y = __uint_as_float((u32)__builtin_amdgcn_readlane((i32)__float_as_uint(given), (int)g));
        u32 more = 0;
        ranked(tk, y, [&](auto is) {
#pragma unroll
          for (u32 j = 0; j < LP_VALS; ++j) more += (u32)__popcll(__ballot(is(j)));
        }, [&](u32 n) { more += n; });
        before += lane == g ? more : 0u;
      }
    }
    if constexpr (TOP) {
      auto append = [&](u32 j, bool take) {
        const u64 mask = __ballot(take);
        if (!mask) return;
        if (take) cand[n + lp_below(mask)] = lp_key(x[j], id(j));
        n += (u32)__popcll(mask);
      };
      if (tile == tile0) {
#pragma unroll
        for (u32 j = 0; j < LP_VALS; ++j) append(j, valid(j) && lp_ordered(x[j]) >= over);
      } else if (__ballot(most > over)) {
#pragma unroll
        for (u32 j = 0; j < LP_VALS; ++j) append(j, x[j] > over);
      }
      if (n > LP_FEW) over = lp_value(lp_thin(cand, n, a.k));
    }
  }
  if (a.given == 1) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) before += (u32)__shfl_xor((int)before, o);
  }
  // the workgroup's: sums of its waves, keys ranked
  sum.s = lp_wave_sum(sum.s); sum.t = lp_wave_sum(sum.t);
  if (lane == 0) { sh.m[w] = sum.m; sh.s[w] = sum.s; sh.t[w] = sum.t; }
  if (lane < a.given) sh.before[w][lane] = before;
  __syncthreads();
  sum = {sh.m[0], sh.s[0], sh.t[0]};
#pragma unroll
  for (u32 i = 1; i < LP_WAVES; ++i) sum.add({sh.m[i], sh.s[i], sh.t[i]}, c);
  if (lane < a.given) {
    before = 0;
#pragma unroll
    for (u32 i = 0; i < LP_WAVES; ++i) before += sh.before[i][lane];
  }
  // the first k of all waves' lists, in order, into top; 0 behind them
  auto first_k = [&]() {
    if (lane < 8) cand[n + lane] = 0;
    if (lane == 0) sh.n[w] = n;
    if (threadIdx.x < LP_MOST) sh.top[threadIdx.x] = 0;
    __syncthreads();
    u32 m = n;
    if (sh.n[0] + sh.n[1] + sh.n[2] + sh.n[3] > LP_RANKED) {         // too many to rank all of them: those that are not below a bound
      u32 best = 0;
#pragma unroll 1
      for (u32 i = lane; i < n; i += 64) best = max(best, (u32)(cand[i] >> 32));
      lp_kth(sh, best, a.k);
      m = 0;
      const u32 kth = sh.kth;
#pragma unroll 1
      for (u32 i = lane; i - lane < n; i += 64) {
        const u64 x = i < n ? cand[i] : 0, mask = __ballot(x && (u32)(x >> 32) >= kth);
        if (x && (u32)(x >> 32) >= kth) cand[m + lp_below(mask)] = x;
        m += (u32)__popcll(mask);
      }
      if (lane < 8) cand[m + lane] = 0;
      if (lane == 0) sh.n[w] = m;
      __syncthreads();
    }
#pragma unroll 1
    for (u32 i = lane; i < m; i += 64) {
      const u64 key = cand[i];
      u32 place = 0;
#pragma unroll 1
      for (u32 l = 0; l < LP_WAVES; ++l) {
        const u64* const x = sh.cand + l * LP_CAP;
        const u32 end = sh.n[l];
#pragma unroll 1
        for (u32 j = 0; j < end; j += 8) {
#pragma unroll
          for (u32 h = 0; h < 8; ++h) place += x[j + h] > key ? 1u : 0u;
        }
      }
      if (place < a.k && key) sh.top[place] = key;
    }
    __syncthreads();
  };
  if constexpr (TOP) first_k();
  if (a.parts > 1) {
    // a part's result past the caches (other workgroups' caches are not this one's); the last part to come adds them up, in their order
    const u32 words = lp_words(a.given, a.k), key0 = lp_key_word(a.given);
    u32* const mine = a.results + (u64)wg * words;
    auto put = [&](u32 i, u32 v) { __hip_atomic_store(mine + i, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
    if (threadIdx.x == 0) { put(0, __float_as_uint(sum.m)); put(1, __float_as_uint(sum.s)); put(2, __float_as_uint(sum.t)); }
    if (threadIdx.x < a.given) put(4 + threadIdx.x, before);
    if (TOP && threadIdx.x < a.k) __hip_atomic_store((u64*)(mine + key0) + threadIdx.x, sh.top[threadIdx.x], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
      const bool last = __hip_atomic_fetch_add(a.ctr + row, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.parts - 1;
      if (last) __hip_atomic_store(a.ctr + row, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      sh.last = last;
    }
    __syncthreads();
    if (!sh.last) return;
    const u32* const all = a.results + (u64)row * a.parts * words;
    auto get = [&](u32 p, u32 i) { return __hip_atomic_load(all + (u64)p * words + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
    if constexpr (TOP) {
      // (a quarter of the keys a wave)
      const u32 per = (a.parts * a.k + LP_WAVES - 1) / LP_WAVES, i0 = min(w * per, a.parts * a.k), i1 = min(i0 + per, a.parts * a.k);
      n = i1 - i0;
      for (u32 i = lane; i < n; i += 64) {
        const u32 p = (i0 + i) / a.k;
        cand[i] = __hip_atomic_load((const u64*)(all + (u64)p * words + key0) + (i0 + i - p * a.k), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
    }
    sum = {-INFINITY, 0.f, 0.f};                     // (a lane a part)
    if (lane < a.parts) sum = {__uint_as_float(get(lane, 0)), __uint_as_float(get(lane, 1)), __uint_as_float(get(lane, 2))};
    if (threadIdx.x < a.given) {
      before = 0;
#pragma unroll 1
      for (u32 p = 0; p < a.parts; p += 8) {         // (eight on their way)
        u32 v[8];
#pragma unroll
        for (u32 i = 0; i < 8; ++i) v[i] = get(min(p + i, a.parts - 1), 4 + threadIdx.x);
#pragma unroll
        for (u32 i = 0; i < 8; ++i) before += p + i < a.parts ? v[i] : 0u;
      }
    }
    sum.to(lp_wave_max(sum.m), c);
    sum.s = lp_wave_sum(sum.s); sum.t = lp_wave_sum(sum.t);
    if constexpr (TOP) first_k();
  }
  const float log_sum = log2f(sum.s), M = sum.m * c;
  auto logprob = [&](float x) {
    const float y = LpSums::near(M) ? __builtin_fmaf(x, c, -M) : (x - sum.m) * c;
    return y == -INFINITY ? (x - sum.m) * inverse - LP_LN2 * log_sum : LP_LN2 * (y - log_sum);      // (a mask's lowest value may overflow in y)
  };
  if (threadIdx.x == 0 && a.entropy) a.entropy[row] = LP_LN2 * (log_sum - sum.t / sum.s);
  if (threadIdx.x < a.given) {
    a.logprobs[(u64)row * a.given + threadIdx.x] = token < 0 ? 0.f : logprob(given);
    if (a.ranks) a.ranks[(u64)row * a.given + threadIdx.x] = token < 0 ? -1 : (i32)before;
  }
  if (TOP && threadIdx.x < a.k) {
    const u64 key = sh.top[threadIdx.x];
    a.top_ids[(u64)row * a.k + threadIdx.x] = (i32)lp_id(key);
    a.top_logprobs[(u64)row * a.k + threadIdx.x] = logprob(lp_value((u32)(key >> 32)));
  }
}
