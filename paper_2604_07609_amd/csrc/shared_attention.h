// Attention of a batch in which the sequences of a group have their first blocks in common (views, and who has which part of the work: paged_views.h;
// the groups' shared keys: paged_attention.h): the parts put together, and the results joined.
#pragma once
#include "paged_attention.h"

// inclusive prefix sum over the wave, without LDS: sums over rows of 16 lanes, then the rows before
__device__ __forceinline__ u32 wave_sums_dpp(u32 v) {
  v += (u32)__builtin_amdgcn_update_dpp(0, (i32)v, 0x111, 0xF, 0xF, true);      // row_shr 1, 2, 4, 8
  v += (u32)__builtin_amdgcn_update_dpp(0, (i32)v, 0x112, 0xF, 0xF, true);
  v += (u32)__builtin_amdgcn_update_dpp(0, (i32)v, 0x114, 0xF, 0xF, true);
  v += (u32)__builtin_amdgcn_update_dpp(0, (i32)v, 0x118, 0xF, 0xF, true);
  v += (u32)__builtin_amdgcn_update_dpp(0, (i32)v, 0x142, 0xA, 0xF, false);     // row_bcast 15 to rows 1 and 3, 31 to rows 2 and 3
  v += (u32)__builtin_amdgcn_update_dpp(0, (i32)v, 0x143, 0xC, 0xF, false);
  return v;
}
// Views; items of the prompts before each sequence (pre) and units of the shared keys before each group (flat); sum[0]: cost of all tiles of few rows, sum[1]: of the prompts.
template <bool BY_MEAN>
__device__ __forceinline__ void views_and_sums(SharedArgs& a, SharedRoom& sh) {
  constexpr u32 NT = 64 * PAGED_WAVES;
  const u32 lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  shared_views<NT, BY_MEAN>(a, (u32*)sh.ring, sh.view);
  if (BY_MEAN) a.short_rows = (u32)__builtin_amdgcn_readfirstlane(a.short_rows);
  u32 (*const of_wave)[4] = (u32(*)[4])sh.ring;
  u32 base[4] = {0, 0, 0, 0};
  for (u32 s0 = 0; s0 < n_views(a); s0 += NT) {
    const u32 s = s0 + threadIdx.x;
    u32 v[4] = {0, 0, 0, 0};
    if (s < n_views(a)) view_units(a, sh.view[s], s >= a.n_seqs, v);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = wave_sums_dpp(v[k]);
    if (s0) __syncthreads();
    if (lane == 63) *(uint4*)of_wave[w] = make_uint4(v[0], v[1], v[2], v[3]);
    __syncthreads();
#pragma unroll
    for (u32 i = 0; i < PAGED_WAVES; ++i) {
      const uint4 x = *(const uint4*)of_wave[i];
      if (i < w) { v[0] += x.x; v[1] += x.y; }
      base[2] += x.z; base[3] += x.w;
      if (i == PAGED_WAVES - 1) {
        if (s < a.n_seqs) sh.pre[s + 1] = base[0] + v[0];
        else if (s < n_views(a)) sh.flat[s - a.n_seqs + 1] = base[1] + v[1];
      }
    }
#pragma unroll
    for (u32 i = 0; i < PAGED_WAVES; ++i) { base[0] += of_wave[i][0]; base[1] += of_wave[i][1]; }
  }
  if (threadIdx.x == 0) { sh.pre[0] = 0; sh.flat[0] = 0; sh.sum[0] = base[2]; sh.sum[1] = base[3]; }
  __syncthreads();
}
template <bool BY_MEAN>
__device__ __forceinline__ SharedWork shared_work(SharedArgs& a, SharedRoom& sh, u32 wg, u32 nwg) {
  constexpr u32 NT = 64 * PAGED_WAVES;
  views_and_sums<BY_MEAN>(a, sh);
  const u32 units = (u32)__builtin_amdgcn_readfirstlane(sh.flat[a.n_groups]);
  const u32 tiles = (u32)__builtin_amdgcn_readfirstlane(sh.sum[0]), prompts = (u32)__builtin_amdgcn_readfirstlane(sh.sum[1]);
  const SharedWork r = deal_out(a, units, tiles, prompts, nwg);
  if (wg == 0 && threadIdx.x == 0) *(u32*)(a.tokens + a.n_tokens) = r.quota;
  // (the parts of prompt items: as the workgroups that take them cut them)
  const u32 item_rows = (u32)__builtin_amdgcn_readfirstlane(sh.pre[a.n_seqs]), parts = prompt_parts(a, item_rows * a.nkv, nwg - r.flat_wgs);
  for (u32 t = wg * NT + threadIdx.x; t < a.n_tokens; t += nwg * NT) a.tokens[t] = join_token(a, sh.view, sh.pre, sh.flat, parts, t);
  __syncthreads();
  return r;
}

// Results joined: of rows whose keys are their group's and their sequence's, and of rows whose keys were cut into parts. A wave per token and as many query heads
// as it has HD / 4 lanes for.
template <int HD> __host__ __device__ constexpr u32 join_heads() { return 64 / (HD / 4); }
template <int HD>
__device__ __forceinline__ void shared_join(const SharedArgs& a, u32 i) {
  constexpr u32 LANES = HD / 4, AT_ONCE = 8;
  const u32 per = (a.nq + join_heads<HD>() - 1) / join_heads<HD>(), lane = threadIdx.x & 63, d = lane % LANES * 4;
  const u32 t = i / per, head = i % per * join_heads<HD>() + lane / LANES, g = head / a.G, h = head - g * a.G;
  if (t >= a.n_tokens) return;
  const JoinToken j = a.tokens[t];
  if (!j.kind) return;
  const u32 quota = *(const u32*)(a.tokens + a.n_tokens);
  if (head < a.nq) {
    float M = -INFINITY, L = 0.f;
    floatx4_t O = {0.f, 0.f, 0.f, 0.f};
    // n results, result(x): maximum and sum, output
    auto take = [&](u32 n, auto ml, auto out) {
      for (u32 x = 0; x < n; x += AT_ONCE) {
        float2 v[AT_ONCE];
        floatx4_t o[AT_ONCE];
#pragma unroll
        for (u32 b = 0; b < AT_ONCE; ++b) {
          v[b] = make_float2(-INFINITY, 0.f);
          o[b] = floatx4_t{0.f, 0.f, 0.f, 0.f};
          if (x + b < n) { v[b] = *(const float2*)ml(x + b); o[b] = *(const floatx4_t*)out(x + b); }
        }
        float mn = M;
#pragma unroll
        for (u32 b = 0; b < AT_ONCE; ++b) mn = fmaxf(mn, v[b].x);
        const float ref = mn == -INFINITY ? 0.f : mn, f = __builtin_amdgcn_exp2f(M - ref);
        L *= f; O *= f;
#pragma unroll
        for (u32 b = 0; b < AT_ONCE; ++b) {
          const float k = __builtin_amdgcn_exp2f(v[b].x - ref);
          L += v[b].y * k;
          O += o[b] * k;
        }
        M = mn;
      }
    };
    auto of_row = [&](u32 which) {
      const float* const b = row_result<HD>(a, which, j.rows[which], head);
      take(1, [&](u32) { return b; }, [&](u32) { return b + 4 + d; });
    };
    if (j.kind == 1) {
      const u32 begin = j.units[0] + g * j.units[1], w0 = begin / quota, w1 = (begin + j.units[2] - 1) / quota, r = j.row + h;
      if (w0 == w1) of_row(0);
      else {
        auto slot = [&](u32 x) { return a.prompt_part + (u64)flat_slot(w0 + x, x == 0) * PROMPT_SLOT(HD); };
        take(w1 - w0 + 1, [&](u32 x) { return slot(x) + 2 * r; }, [&](u32 x) { return slot(x) + 2 * PROMPT_ROWS + r * HD + d; });
      }
    }
    if (j.parts > 1) {
      const u32 r = j.own_row + h, item = (j.top - r / PROMPT_ROWS) * a.nkv + g, in = r % PROMPT_ROWS;
      const float* const first = a.own_part + (u64)item * j.parts * PROMPT_SLOT(HD);
      take(j.parts, [&](u32 x) { return first + (u64)x * PROMPT_SLOT(HD) + 2 * in; }, [&](u32 x) { return first + (u64)x * PROMPT_SLOT(HD) + 2 * PROMPT_ROWS + in * HD + d; });
    } else of_row(1);
    const float inv = L == 0.f ? 0.f : 1.0f / L;
    *(uint2*)out_at(a, t, head * HD + d) = make_uint2(half_pair(O[0] * inv, O[1] * inv), half_pair(O[2] * inv, O[3] * inv));
  }
}

// The tiles of few rows: views from where the prompt part has them to where the few-row part does, then that part. It has eight waves here, also with one row tile over 4 bits, where three
// workgroups of four on a compute unit are 7 to 13 % faster (SHORT_SMALL): the prompt part's ring leaves LDS for one workgroup.
template <int HD, int BITS, int CT>
__device__ __forceinline__ void few_rows(const SharedArgs& a, const SharedRoom& p, ShortShared<HD, CT, PAGED_WAVES, true>& sh, u32 wg, u32 nwg) {
  constexpr u32 NT = 64 * PAGED_WAVES;
  SharedView v[PAGED_MAX_SEQS / NT];
#pragma unroll
  for (u32 j = 0; j < PAGED_MAX_SEQS / NT; ++j) if (threadIdx.x + j * NT < n_views(a)) v[j] = p.view[threadIdx.x + j * NT];
  __syncthreads();
#pragma unroll
  for (u32 j = 0; j < PAGED_MAX_SEQS / NT; ++j) {
    const u32 s = threadIdx.x + j * NT;
    if (s >= n_views(a)) continue;
    const bool group = s >= a.n_seqs;
    sh.pos0[s] = v[j].pos0;
    sh.n[s] = short_unit_count(a, v[j], group) ? (unsigned char)v[j].n : (unsigned char)0;
    sh.link[s] = group ? (uint16_t)v[j].row() : v[j].first ? (uint16_t)v[j].group() : (uint16_t)NO_GROUP;
  }
  __syncthreads();
  paged_short<HD, BITS, CT, SHORT_AHEAD(HD, BITS, CT), PAGED_WAVES>(a, sh, wg, nwg);
}
// A call with groups. A row's keys are its group's and its own: softmax((s1, s2)) v is joined from each part's maximum m, sum l and output o about m, by
// o = (2^(m1-M) o1 + 2^(m2-M) o2) / (2^(m1-M) l1 + 2^(m2-M) l2). With n members of g rows each the shared keys are read once and not n times, and are products of n g rows:
// what was bound by bytes becomes bound by products, while the members' own keys stay bound by bytes. So some workgroups have the groups' shared keys, others at the same time
// the tiles of few rows, as many each as their estimated times ask for, and whoever is done takes the prompts' items (with one run of all shared keys, and no item behind it, 32 sequences behind
// 4000 tokens beside a prompt of 8192 took 737 us, so 591, every sequence by itself 628). One after the other on all workgroups: 158 us, so 99, for 253 sequences
// behind 8200 tokens with 17 to 1000 of their own; bytes of all keys that are there 58 us, every sequence by itself 1000.
// Of a call's time 3 to 5 us are the views and sums, 4 to 9 the join (a kernel of its own: results of other workgroups are in memory behind it), a workgroup's start and end 5.
// CT: row tiles of the few-row part; ANY_CT: one, or SHORT_MORE, by the views (both instances in one kernel: within 1 us of one alone; the larger one for all calls took 51 and not 40 us for three
// groups of 30, heads of 64 over 4 bits). Of scalar registers 175 to 292 are spilled, into vector registers, and not in the loops over tiles or steps as far as arguments loaded anew can help it; with
// heads of 64 over 4 bits 3 vector registers to memory.
#define ANY_CT 0
template <int HD, int CT> union SharedKernelRoom { ShortShared<HD, CT, PAGED_WAVES, true> s; SharedRoom p; };
template <int HD> union SharedKernelRoom<HD, ANY_CT> { ShortShared<HD, 1, PAGED_WAVES, true> one; ShortShared<HD, SHORT_MORE(HD), PAGED_WAVES, true> more; SharedRoom p; };
template <int HD, int BITS, int CT>
__device__ __forceinline__ void shared_attention(const SharedArgs& args, SharedKernelRoom<HD, CT>& sh, u32 wg, u32 nwg) {
  constexpr bool BY_MEAN = CT == ANY_CT;
  SharedArgs mine = args;
  const SharedWork work = shared_work<BY_MEAN>(mine, sh.p, wg, nwg);
  const u32 short_rows = mine.short_rows;
  auto part_args = [&]() { SharedArgs a = fresh_args(); if (BY_MEAN) a.short_rows = short_rows; return a; };
  if (wg < work.flat_wgs) {
    const SharedArgs a = part_args();
    const u32 units = (u32)__builtin_amdgcn_readfirstlane(sh.p.flat[a.n_groups]), from = min(wg * work.quota, units);
    paged_prompt<HD, BITS, true>(a, sh.p, wg, work.flat_wgs, false, FlatRun{from, min(from + work.quota, units)});
  } else if (work.few) {
    const SharedArgs a = part_args();
    const u32 few_wg = wg - work.flat_wgs, few_wgs = nwg - work.flat_wgs;
    if constexpr (CT != ANY_CT) few_rows<HD, BITS, CT>(a, sh.p, sh.s, few_wg, few_wgs);
    else if (short_rows == 16) few_rows<HD, BITS, 1>(a, sh.p, sh.one, few_wg, few_wgs);
    else few_rows<HD, BITS, SHORT_MORE(HD)>(a, sh.p, sh.more, few_wg, few_wgs);
  }
  if (!work.prompts) return;
  SharedArgs a = part_args();
  __syncthreads();
  if (work.few && wg >= work.flat_wgs) views_and_sums<BY_MEAN>(a, sh.p);
  paged_prompt<HD, BITS>(a, sh.p, wg, nwg, true, FlatRun{0, 0}, nwg - work.flat_wgs);
}
