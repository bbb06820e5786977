// Log probabilities of given tokens with their ranks, the entropy and the most probable tokens, from rows of logits that are read once.
// With z = x * inverse temperature, m the row's maximum and S = sum exp(z - m): log p = z - m - log S, entropy = log S - sum (z - m) exp(z - m) / S.
// Both sums are of y = (x - m) c, c = inverse temperature * log2(e), and 2^y: y 2^y is at most 0.54 whatever the temperature. Every lane keeps its own running maximum and sums of the logits it reads, so nobody waits for anybody until the end.
//
// Order: larger logits first, of equal ones the lower id; a key of 64 bits (the logit's bits turned into a whole number, then the id
// downwards) makes every place of it distinct. The k first ones of a tile: the lanes' largest keys, in groups of neighbouring lanes, are ranked
// against each other; at least k logits are not below the kth of them, T, and those are in the k groups whose largest are not, so they are
// few and fit in LDS whatever the row holds. Later tiles add what is above T. What comes together is thinned out the same way and at last ranked,
// every key against every other.
#pragma once
#include "blink_device.h"

#define LP_VALS 32u                // logits of a lane in a tile
#define LP_TILE (BLK_THREADS * LP_VALS)
#define LP_MOST 64u                // given tokens, most probable tokens
#define LP_NEW (LP_MOST * LP_VALS) // keys that a tile adds at most once T is its own
#define LP_FEW 512u                // keys that are ranked as they are
#define LP_CAP (LP_FEW + LP_NEW)
#define LP_MAX_PARTS 32u           // workgroups of a row (LP_MAX_PARTS LP_MOST keys at most are joined)
#define LP_PER_CU 4u               // workgroups that a call has for every compute unit, where its rows have the tiles
#define LP_LOWEST -3.4028235e38f
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
// a part's result: maximum and sums, logits before each given one, then keys
__host__ __device__ __forceinline__ u32 lp_key_word(u32 given) { return (4 + given + 1) & ~1u; }
__host__ __device__ __forceinline__ u32 lp_words(u32 given, u32 k) { return lp_key_word(given) + 2 * k; }

struct LogprobShared {
  u64 cand[LP_CAP], spare[LP_MOST * ((LP_CAP + BLK_THREADS - 1) / BLK_THREADS)], group[BLK_THREADS], top[LP_MOST], T;
  u32 cnt[BLK_THREADS], n, last;
  float m[4], s[4], t[4], given[LP_MOST];
  i32 token[LP_MOST];
  u32 before[LP_MOST];
};

__device__ __forceinline__ float lp_ordered(float x) { return fmaxf(x, -INFINITY); }      // NaN: as -inf
__device__ __forceinline__ u64 lp_key(float x, u32 id) {
  const u32 b = __float_as_uint(lp_ordered(x) + 0.0f);                                    // (-0: as 0)
  return (u64)(b ^ ((i32)b < 0 ? 0xFFFFFFFFu : 0x80000000u)) << 32 | (0xFFFFFFFFu - id);
}
__device__ __forceinline__ u32 lp_id(u64 key) { return 0xFFFFFFFFu - (u32)key; }
__device__ __forceinline__ float lp_value(u64 key) { const u32 u = (u32)(key >> 32); return __uint_as_float(u ^ ((i32)u < 0 ? 0x80000000u : 0xFFFFFFFFu)); }
__device__ __forceinline__ u64 lp_shfl_xor(u64 v, int o) { return (u64)(u32)__shfl_xor((int)(v >> 32), o) << 32 | (u32)__shfl_xor((int)v, o); }

// The kth largest of the groups' largest keys (0: there are fewer), n = BLK_THREADS / lanes groups; `mine`: the lane's largest key.
__device__ __forceinline__ u64 lp_kth(LogprobShared& sh, u64 mine, u32 k, u32 lanes) {
  for (u32 o = 1; o < lanes; o <<= 1) { const u64 x = lp_shfl_xor(mine, (int)o); mine = x > mine ? x : mine; }
  const u32 n = BLK_THREADS / lanes, i = threadIdx.x & (n - 1), per = n * n / BLK_THREADS;
  __syncthreads();
  if (threadIdx.x % lanes == 0) sh.group[threadIdx.x / lanes] = mine;
  sh.cnt[threadIdx.x] = 0;
  if (threadIdx.x == 0) sh.T = 0;
  __syncthreads();
  const u64 key = sh.group[i];
  if (per) {                                         // every lane a part of the comparisons
    const u32 j0 = threadIdx.x / n * per;
    u32 c = 0;
    for (u32 j = j0; j < j0 + per; ++j) c += sh.group[j] > key ? 1u : 0u;
    if (c) atomicAdd(&sh.cnt[i], c);
  } else if (threadIdx.x < n * n && sh.group[threadIdx.x / n] > key) atomicAdd(&sh.cnt[i], 1u);
  __syncthreads();
  if (threadIdx.x < n && sh.cnt[threadIdx.x] == k - 1 && key) sh.T = key;
  __syncthreads();
  return sh.T;
}
// The min(k, n) largest of cand[0 .. n), in order, into top; 0 behind them.
__device__ __forceinline__ void lp_select(LogprobShared& sh, u32 n, u32 k) {
  while (n > LP_FEW) {
    u64 best = 0;
    for (u32 i = threadIdx.x; i < n; i += BLK_THREADS) best = sh.cand[i] > best ? sh.cand[i] : best;
    const u64 T = lp_kth(sh, best, k, 1);
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    for (u32 i = threadIdx.x; i < n; i += BLK_THREADS)
      if (sh.cand[i] >= T) sh.spare[atomicAdd(&sh.n, 1u)] = sh.cand[i];      // (of k lanes)
    __syncthreads();
    n = sh.n;
    for (u32 i = threadIdx.x; i < n; i += BLK_THREADS) sh.cand[i] = sh.spare[i];
    __syncthreads();
  }
  __syncthreads();
  if (threadIdx.x < k) sh.top[threadIdx.x] = 0;
  __syncthreads();
  for (u32 i = threadIdx.x; i < n; i += BLK_THREADS) {
    const u64 key = sh.cand[i];
    u32 c = 0;
    for (u32 j = 0; j < n; ++j) c += sh.cand[j] > key ? 1u : 0u;
    if (c < k) sh.top[c] = key;
  }
  __syncthreads();
}

struct LpSums {
  float m, s, t;                                     // maximum, sum 2^y, sum y 2^y of y = (x - m) c
  __device__ __forceinline__ void to(float mn, float c) {      // the same with mn >= m for the maximum
    if (m == -INFINITY) { m = mn; return; }          // (nothing yet: sums of 0, or NaN)
    const float y = (m - mn) * c, f = __builtin_amdgcn_exp2f(y);
    t = f > 0.f ? f * __builtin_fmaf(y, s, t) : 0.f; // (y may be -inf)
    s *= f;
    m = mn;
  }
  __device__ __forceinline__ void add(float m2, float s2, float t2, float c) {
    LpSums o = {m2, s2, t2};
    const float mn = fmaxf(m, m2);
    to(mn, c); o.to(mn, c);
    s += o.s; t += o.t;
  }
};

template <typename T>
__device__ __forceinline__ void lp_load(float (&x)[LP_VALS], const T* base, u32 at, u32 begin, u32 end, bool whole) {
  constexpr u32 VEC = 16 / sizeof(T), NV = LP_VALS / VEC;
  typedef T vec_t __attribute__((ext_vector_type(VEC)));
#pragma unroll
  for (u32 v = 0; v < NV; ++v) {
    const u32 i = at + (v * BLK_THREADS + threadIdx.x) * VEC;
    if (whole || (i >= begin && i + VEC <= end)) {
      const vec_t y = __builtin_nontemporal_load((const vec_t*)(base + i));
#pragma unroll
      for (u32 j = 0; j < VEC; ++j) x[v * VEC + j] = (float)y[j];
    } else {
#pragma unroll
      for (u32 j = 0; j < VEC; ++j) x[v * VEC + j] = i + j >= begin && i + j < end ? (float)base[i + j] : -INFINITY;
    }
  }
}

template <typename T, bool TOP>
__device__ __forceinline__ void token_logprobs(const LogprobArgs& a, LogprobShared& sh, u32 wg) {
  constexpr u32 VEC = 16 / sizeof(T);
  const u32 row = wg / a.parts, part = wg - row * a.parts, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  // the row's elements are [shift, end) of what begins at the 16 bytes its first one lies in
  const T* const first = (const T*)a.x + (u64)row * a.stride;
  const u32 shift = (u32)((u64)first % 16 / sizeof(T)), end = shift + a.V;
  const T* const base = first - shift;
  const u32 tiles = (end + LP_TILE - 1) / LP_TILE, tile0 = (u32)((u64)tiles * part / a.parts), tile1 = (u32)((u64)tiles * (part + 1) / a.parts);
  const float inverse = a.inverse ? a.inverse[row] : 1.f;
  float c = inverse * 1.44269504088896340736f;
  if (!(inverse > 0.f) || !(c < INFINITY)) c = __uint_as_float(0x7FC00000u);
  if (threadIdx.x < a.given) {
    const i32 t = a.tokens[(u64)row * a.given + threadIdx.x];
    const bool in = t >= 0 && (u32)t < a.V;
    sh.token[threadIdx.x] = in ? t : -1;
    sh.given[threadIdx.x] = in ? lp_ordered((float)first[t]) : 0.f;
    sh.before[threadIdx.x] = 0;
  }
  if (threadIdx.x == 0) sh.n = 0;
  __syncthreads();
  LpSums sum = {-INFINITY, 0.f, 0.f};
  u32 lanes = 1;                                     // of a group, so that no tile adds more than LP_NEW keys
  while (TOP && 2 * lanes * a.k <= LP_MOST) lanes *= 2;
  u64 least = 0;                                     // k keys at least are not below this one
  float over = 0.f;                                  // its logit
  u32 n = 0;                                         // keys in cand
#pragma unroll 1
  for (u32 tile = tile0; tile < tile1; ++tile) {
    const u32 at = tile * LP_TILE;
    const bool whole = at >= shift && at + LP_TILE <= end;
    float x[LP_VALS];
    lp_load<T>(x, base, at, shift, end, whole);
    auto id = [&](u32 j) { return at + (j / VEC * BLK_THREADS + threadIdx.x) * VEC + j % VEC - shift; };
    auto valid = [&](u32 j) { return whole || id(j) < a.V; };      // (before the row: beyond 2^31)
    float most = -INFINITY;
#pragma unroll
    for (u32 j = 0; j < LP_VALS; ++j) most = fmaxf(most, x[j]);
    sum.to(fmaxf(sum.m, most), c);
    const float ref = sum.m == -INFINITY ? 0.f : sum.m;
#pragma unroll
    for (u32 j = 0; j < LP_VALS; ++j) {
      const float y = (x[j] - ref) * c, e = __builtin_amdgcn_exp2f(y);
      sum.s += e;
      sum.t = __builtin_fmaf(fmaxf(y, LP_LOWEST), e, sum.t);         // (0 times -inf is to be 0)
    }
    if (a.ranks) {
#pragma unroll 1
      for (u32 g = 0; g < a.given; ++g) {
        const u32 t = (u32)__builtin_amdgcn_readfirstlane(sh.token[g]);
        const float y = __uint_as_float((u32)__builtin_amdgcn_readfirstlane((i32)__float_as_uint(sh.given[g])));
        u32 before = 0;
        if (!whole || (t + shift >= at && t + shift < at + LP_TILE)) {
#pragma unroll
          for (u32 j = 0; j < LP_VALS; ++j) { const float o = lp_ordered(x[j]); before += (u32)__popcll(__ballot(valid(j) && (o > y || (o == y && id(j) < t)))); }
        } else if (t + shift < at) {
#pragma unroll
          for (u32 j = 0; j < LP_VALS; ++j) before += (u32)__popcll(__ballot(x[j] > y));
        } else {
#pragma unroll
          for (u32 j = 0; j < LP_VALS; ++j) before += (u32)__popcll(__ballot(lp_ordered(x[j]) >= y));
        }
        if (lane == 0) atomicAdd(&sh.before[g], before);
      }
    }
    if constexpr (TOP) {
      // the keys of this tile that `take` names, behind the first n of cand; how many there are then (more than fit: none of the rest is there)
      auto append = [&](auto take) {
        u32 mine = 0;
#pragma unroll
        for (u32 j = 0; j < LP_VALS; ++j) mine += take(j) ? 1u : 0u;
        if (mine) {
          u32 to = atomicAdd(&sh.n, mine);
#pragma unroll
          for (u32 j = 0; j < LP_VALS; ++j)
            if (take(j)) { if (to < LP_CAP) sh.cand[to] = lp_key(x[j], id(j)); ++to; }
        }
        __syncthreads();
        return sh.n;
      };
      u32 now = LP_CAP + 1;
      if (tile != tile0) now = append([&](u32 j) { return x[j] > over; });      // (equal ones have the higher ids)
      if (now > LP_CAP) {
        u64 best = 0;
#pragma unroll
        for (u32 j = 0; j < LP_VALS; ++j)
          if (lp_ordered(x[j]) == most && valid(j) && !best) best = lp_key(x[j], id(j));
        const u64 kth = lp_kth(sh, best, a.k, lanes);
        least = kth > least ? kth : least;
        over = lp_value(least);
        if (threadIdx.x == 0) sh.n = n;
        __syncthreads();
        now = append([&](u32 j) { return valid(j) && lp_key(x[j], id(j)) >= least; });
      }
      n = now;
      if (n > LP_FEW && tile + 1 < tile1) {
        lp_select(sh, n, a.k);
        n = a.k;
        for (u32 i = threadIdx.x; i < n; i += BLK_THREADS) sh.cand[i] = sh.top[i];
        least = sh.top[a.k - 1];
        over = lp_value(least);
        if (threadIdx.x == 0) sh.n = n;
      }
      __syncthreads();                               // (before the next tile adds to sh.n)
    }
  }
  // the workgroup's sums
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) sum.add(__shfl_xor(sum.m, o), __shfl_xor(sum.s, o), __shfl_xor(sum.t, o), c);
  if (lane == 0) { sh.m[w] = sum.m; sh.s[w] = sum.s; sh.t[w] = sum.t; }
  if constexpr (TOP) lp_select(sh, n, a.k);
  __syncthreads();
  sum = {sh.m[0], sh.s[0], sh.t[0]};
#pragma unroll
  for (int i = 1; i < 4; ++i) sum.add(sh.m[i], sh.s[i], sh.t[i], c);
  if (a.parts > 1) {
    // a part's result past the caches (other workgroups' caches are not this one's); the last part to come adds them up, in their order
    const u32 words = lp_words(a.given, a.k), key0 = lp_key_word(a.given);
    u32* const mine = a.results + (u64)wg * words;
    auto put = [&](u32 i, u32 v) { __hip_atomic_store(mine + i, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
    if (threadIdx.x == 0) { put(0, __float_as_uint(sum.m)); put(1, __float_as_uint(sum.s)); put(2, __float_as_uint(sum.t)); }
    if (threadIdx.x < a.given) put(4 + threadIdx.x, sh.before[threadIdx.x]);
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
    // (a lane a part, added up as the lanes of a wave are)
    sum = {-INFINITY, 0.f, 0.f};
    if (lane < a.parts) sum = {__uint_as_float(get(lane, 0)), __uint_as_float(get(lane, 1)), __uint_as_float(get(lane, 2))};
    if (threadIdx.x < a.given) {
      u32 before = 0;
      for (u32 p = 0; p < a.parts; ++p) before += get(p, 4 + threadIdx.x);
      sh.before[threadIdx.x] = before;
    }
    if constexpr (TOP) {
      n = a.parts * a.k;
      for (u32 i = threadIdx.x; i < n; i += BLK_THREADS)
        sh.cand[i] = __hip_atomic_load((const u64*)(all + (u64)(i / a.k) * words + key0) + i % a.k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) sum.add(__shfl_xor(sum.m, o), __shfl_xor(sum.s, o), __shfl_xor(sum.t, o), c);
    __syncthreads();
    if constexpr (TOP) lp_select(sh, n, a.k);
  }
  const float log_sum = logf(sum.s);
  auto logprob = [&](float x) { return __builtin_fmaf(x - sum.m, inverse, -log_sum); };
  if (threadIdx.x == 0 && a.entropy) a.entropy[row] = log_sum - 0.69314718055994530942f * sum.t / sum.s;
  if (threadIdx.x < a.given) {
    const i32 t = sh.token[threadIdx.x];
    a.logprobs[(u64)row * a.given + threadIdx.x] = t < 0 ? 0.f : logprob(sh.given[threadIdx.x]);
    if (a.ranks) a.ranks[(u64)row * a.given + threadIdx.x] = t < 0 ? -1 : (i32)sh.before[threadIdx.x];
  }
  if (TOP && threadIdx.x < a.k) {
    const u64 key = sh.top[threadIdx.x];
    a.top_ids[(u64)row * a.k + threadIdx.x] = (i32)lp_id(key);
    a.top_logprobs[(u64)row * a.k + threadIdx.x] = logprob(lp_value(key));
  }
}
