// Who has which part of a call's work: the sequences' and the groups' views, and how the groups' shared keys, the rest and the joining of results are dealt out. Whole numbers and
// no more, none of it by lanes or waves, so that it can be gone through on a CPU as well.
#pragma once
#include <type_traits>

// Row tiles of the short part beyond one (64 rows with heads of 64, 32 of 128: what the registers hold; 8 sequences of 4000 keys with 32
// rows take 30 us and 60 as prompts, 30 of 2000 in 4 bits with 40 rows 24 and 47)
#define SHORT_MORE(HD) ((HD) == 64 ? 4 : 2)
#define PAGED_MAX_SEQS 1024u       // sequences (and groups) whose views a workgroup keeps in LDS
#define PROMPT_CT 2u
#define PROMPT_ROWS (128u * PROMPT_CT)
#define SHARED_ROWS 256u           // sequences with so many rows fill a prompt item by themselves
#define FLAT_STEP 4u               // units of a step of the groups' shared keys, and of one of an item of 128 rows or less
#define FLAT_LIGHT 3u
#define SHARED_GAIN 4.f            // units that a group must save for a kv head: its start and end, two times, beside those of others
#define FEW_MORE 1.5f              // time of a tile of few rows in an instance with more than one row tile, in those with one
#define GROUPS_UNIT (1u << 18)     // (more than the queries of all members: 1023 times 255)
#define FEW_PAIR 3u                // what a pair of a sequence and a kv head takes beside its tiles, in tiles (96 sequences with 5 to 300 keys of their own, in 4 bits: 88 us with 2, 81 with 3 and 4; 253 with 17 to 1000: 105 with none, 99 with 1 to 3)
#define NO_GROUP 0xFFFFu

struct PagedArgs {
  const f16_t* q;                 // [token][q head][hd]
  u64 qs;                         // elements between tokens
  f16_t* out;                     // [token][q head][hd], or packed GEMM operand (out_tbs != 0)
  u64 os;
  u32 out_tbs;
  const i32 *cu, *lens;           // first token of every sequence (n_seqs + 1), its context with them
  const u32* tables;              // [row][max_blocks] block ids
  const u32* table_row;           // row of every sequence (null: its number)
  const void* cache;
  u32 n_blocks, max_blocks;
  u32 nq, nkv, G;
  u32 n_seqs, n_tokens, max_q;    // sequences; tokens of q and out; queries of a sequence that are looked at
  u32 window, sinks;
  float c;                        // scale of the scores * log2(e)
  u32 short_rows;                 // sequences with at most so many rows are the short part's (of a call with groups by shared_views, where rows_by_mean)
  u32 n_splits;                   // most parts of a prompt item's keys
  u32* ctr;                       // zeros between launches (paged_counters): next prompt item, workgroups done, then the short part's
  float *part, *prompt_part;      // partial results of the short and of the prompt part
};

// A call in which sequences of a group have their first blocks in common: those keys are seen once for the group, by the rows of all of its
// sequences at a time (shared_views). So a call has a view for each sequence and, behind those, one for each group.
struct SharedArgs : PagedArgs {
  u32 n_groups, share_all;        // share_all: groups that gain nothing by it too
  const i32 *starts, *shared;     // first sequence of every group (n_groups + 1), tokens that its sequences share
  float* rows;                    // results to be joined: [of the group, of the sequence][n_rows][q head] of ROW_RESULT(hd) floats (row_index)
  u32 n_rows, row_tokens;         // a row per token or, where that is less, row_tokens of them per sequence (0: per token)
  float* own_part;                // parts of prompt items (prompt_part: of the groups' items)
  u32 least;                      // units of a step of a group of 32 rows or less in all (of others: FLAT_STEP, of items of 128 rows or less FLAT_LIGHT)
  u32 lead;                       // time of an item of the groups' shared keys beside its steps, in units (FlatShape)
  u32 most_rows;                  // rows that the short part's registers hold
  float few_cost;                 // time of a tile of few rows on one compute unit, in units, with one row tile (with more of them: FEW_MORE times that)
  u32 gain;                       // units that all groups together must save for a kv head
  float row_cost;                 // units that the rows of a member's token, to be joined, take for a kv head
  struct JoinToken* tokens;       // what is to be joined of every token, and behind them the units of a workgroup's run (FlatRun)
};
#define ROW_RESULT(HD) ((HD) + 4u)                   // maximum, sum, two unused, output
template <typename A> constexpr bool is_shared = std::is_same<A, SharedArgs>::value;
__device__ __forceinline__ u32 n_views(const PagedArgs& a) { return a.n_seqs; }
__device__ __forceinline__ u32 n_views(const SharedArgs& a) { return a.n_seqs + a.n_groups; }

// One sequence: its tokens, where its queries stand, and which blocks they see
struct SeqView {
  u32 t0, n;
  i32 pos0;
  __device__ __forceinline__ u32 lo() const { return 0; }
};
// The same, and of a group: the queries of its members, one member's after the other's, t0 the first one's token; all stand at the group's last key. first: the first key seen
// here (those before it are the group's), a multiple of 64
struct SharedView {
  u32 t0, n;
  i32 pos0;
  u32 first, which;
  // of a sequence (first != 0): its group, and how many queries the members of all groups have before it (less than 2^18; there only where some group has gaps)
  __device__ __forceinline__ u32 group() const { return which & (PAGED_MAX_SEQS - 1); }
  __device__ __forceinline__ u32 before() const { return which / PAGED_MAX_SEQS; }
  // of a group: its first member, whose row of the table it takes, and whether tokens of others lie between its members'
  __device__ __forceinline__ u32 row() const { return which & (PAGED_MAX_SEQS - 1); }
  __device__ __forceinline__ bool gaps() const { return which >= PAGED_MAX_SEQS; }
  __device__ __forceinline__ u32 lo() const { return first; }
};
__device__ __forceinline__ SeqView seq_view(const PagedArgs& a, u32 s) {
  SeqView v;
  const i32 c0 = max(0, min(a.cu[s], (i32)a.n_tokens)), c1 = max(c0, min(a.cu[s + 1], (i32)a.n_tokens));
  v.t0 = (u32)c0;
  v.n = min((u32)(c1 - c0), a.max_q);
  v.pos0 = max(0, min(a.lens[s], (i32)(a.max_blocks * 16))) - (c1 - c0);
  return v;
}
// Visible tiles of TK keys of the queries at positions p0 .. p1 (p1 >= 0): the first `zb` ones, then those from `wlo` to `hi`
struct Seen { u32 zb, wlo, n; };
// (lo: keys before this multiple of TK are not looked at; not together with a window that begins behind key 0)
template <u32 TK>
__device__ __forceinline__ Seen seen_tiles(const PagedArgs& a, i32 p0, i32 p1, u32 lo = 0) {
  Seen r;
  r.wlo = a.window && p0 >= (i32)a.window ? (u32)(p0 - (i32)a.window + 1) / TK : 0u;
  r.zb = min((a.sinks + TK - 1) / TK, r.wlo);
  r.wlo += lo / TK;
  r.n = p1 < 0 ? 0u : r.zb + (u32)p1 / TK + 1 - r.wlo;
  return r;
}

// The groups with more rows than the few-row part takes, or with others' tokens between their members' (rows are looked up here, and not there: 60 scalar registers more): their rows in items of
// flat_rows (whole queries), each with all shared keys. All steps of all (group, kv head, item) are one line of units, FLAT_STEP, FLAT_LIGHT or `least` a step, and `lead` ahead of an item's, and every workgroup has an equal run of it. An item inside a run is
// done there; one that several runs share leaves a result in each. The units are what workgroups' times fit, to within 1.3 us of 30 to 75: a piece of an item, its start and end, takes
// 6.3 us (over 4 bits 7.0; with heads of 64: 6.8, 4.4), a step of 256 rows 1.87 (2.25; 1.52, 1.97), one of 128 or less 1.37 (1.68; 1.10, 1.47), of a
// group of 32 rows over halves 1.17, bound by bytes like the tiles of few rows.
__device__ __forceinline__ u32 flat_rows(const PagedArgs& a) { return PROMPT_ROWS / a.G * a.G; }
struct FlatShape {
  u32 items, steps, lead, last;                      // items of a kv head; units of the last one's steps (the others': FLAT_STEP)
  __device__ __forceinline__ u32 units(u32 item) const { return steps * (item + 1 < items ? FLAT_STEP : last) + lead; }
  __device__ __forceinline__ u32 all() const { return (items - 1) * (FLAT_STEP * steps + lead) + last * steps + lead; }
};
__device__ __forceinline__ FlatShape flat_shape(const SharedArgs& a, u32 rows, u32 keys) {
  const u32 per = flat_rows(a), items = (rows + per - 1) / per;
  return {items, keys / 64, a.lead, rows - (items - 1) * per > 128 ? FLAT_STEP : rows > 32 ? FLAT_LIGHT : a.least};
}
__device__ __forceinline__ FlatShape flat_shape(const SharedArgs& a, const SharedView& v) { return flat_shape(a, v.n * a.G, (u32)v.pos0 + 1); }
__device__ __forceinline__ u32 flat_units(const SharedArgs& a, const SharedView& v) {      // of a group
  return v.n * a.G <= a.short_rows && !v.gaps() ? 0u : flat_shape(a, v).all() * a.nkv;
}
// The views of a call with groups, by a workgroup of NT threads, in LDS: those of the sequences, then those of the groups. A sequence goes by its group where it gains by that and may: it has fewer rows than a prompt item,
// all its queries stand behind the shared keys and see every one of them, and all of these together take less time with the shared keys apart; and only if all groups together gain more than
// what results that are joined take. A group's rows are those of its members, wherever in its range of sequences they stand. The shared keys are cut to a multiple of 64, what a step of the
// prompt part takes. room: ROOM_WORDS of LDS.
//
// Row tiles of the few-row part (short_rows): more than one where a sequence needs them, and none needs more than it holds (beside a prompt 96 sequences with 5 drafts, 20 rows, take 149 us as prompt
// items and 169 as two row tiles, in 4 bits 176 and 193), and where the groups' mean does: a step of a prompt item costs a group of few rows as much as one of 128, over 4 bits as one of 256. 40 groups
// of up to four sequences with 9 queries, heads of 64: 67 us with the groups' keys as steps of prompt items, 52 to 57 as tiles of few rows; 16 groups of 8 behind 2000 and 8000 tokens, heads of 64: 41
// and 90, so 32 and 72; heads of 128 over 4 bits: 52 and 132, so 40 and 68, and beside 100 sequences in no group 204 and 156. Over halves with heads of 128 the steps are as fast or faster (46 and
// 117 us, as tiles 47 and 120; behind 500 tokens 31, 36), so there the host says what a call takes, by its longest run of queries, or by all tokens where those are few (shared_costs).
// The mean is that of the groups that there are: lengths are known here only.
#define SPREAD 32u                 // places of a sum that many lanes add to
#define ROOM_WORDS (9 * PAGED_MAX_SEQS + 3 * SPREAD + 16)
constexpr bool rows_by_mean(int hd, int bits) { return hd == 64 || bits == 4; }
template <u32 NT, bool BY_MEAN>
__device__ __forceinline__ void shared_views(SharedArgs& a, u32* room, SharedView* view) {
  constexpr u32 EACH = (PAGED_MAX_SEQS + NT - 1) / NT, OPTIONS = BY_MEAN ? 2 : 1;
  // gained[option], sizes: of all groups, in SPREAD places; whether some group has gaps, some sequence more than 16 rows that the few-row part holds, some more than that. Then of every
  // group: first sequence, shared keys, and of its members: the first one, how many, their queries, first token and last one + 1
  u32 *const gained = room, *const sizes = gained + 2 * SPREAD, *const gaps = sizes + SPREAD, *const some_rows = gaps + 1, *const many_rows = some_rows + 1;
  u32 *const starts = gaps + 8, *const keys = starts + a.n_groups + 1, *const from = keys + a.n_groups, *const members = from + a.n_groups, *const queries = members + a.n_groups;
  u32 *const t0 = queries + a.n_groups, *const t1 = t0 + a.n_groups, *const scratch = t1 + a.n_groups;
  for (u32 i = threadIdx.x; i < 3 * SPREAD + 3; i += NT) room[i] = 0;
  for (u32 g = threadIdx.x; g <= a.n_groups; g += NT) {
    starts[g] = (u32)max(0, min(a.starts[g], (i32)a.n_seqs));
    if (g == a.n_groups) break;
    keys[g] = (u32)max(0, min(a.shared[g], (i32)(a.max_blocks * 16))) / 64 * 64;
    from[g] = t0[g] = ~0u; members[g] = queries[g] = t1[g] = 0;
  }
  SeqView v[EACH];                                   // (asked for before the barrier)
#pragma unroll
  for (u32 j = 0; j < EACH; ++j)
    if (threadIdx.x + j * NT < a.n_seqs) v[j] = seq_view(a, threadIdx.x + j * NT);
  __syncthreads();
  u32 group[EACH];
#pragma unroll
  for (u32 j = 0; j < EACH; ++j) {
    const u32 s = threadIdx.x + j * NT;
    group[j] = NO_GROUP;
    if (s >= a.n_seqs) continue;
    if (BY_MEAN && v[j].n * a.G > 16) *(v[j].n * a.G > a.most_rows ? many_rows : some_rows) = 1;
    if (!a.n_groups || s < starts[0]) continue;
    u32 g = 0;
    for (u32 step = 1u << (31 - __clz((int)a.n_groups)); step; step >>= 1) if (g + step < a.n_groups && starts[g + step] <= s) g += step;      // the last that begins here or before
    const i32 p1 = v[j].pos0 + (i32)v[j].n - 1;
    if (s >= starts[g + 1] || !keys[g] || !v[j].n || v[j].n * a.G >= SHARED_ROWS || v[j].pos0 < (i32)keys[g] || (a.window && p1 >= (i32)a.window)) continue;
    atomicMin(from + g, s);
    atomicAdd(members + g, 1u);
    atomicAdd(queries + g, v[j].n);
    atomicMin(t0 + g, v[j].t0);
    atomicMax(t1 + g, v[j].t0 + v[j].n);
    view[s] = SharedView{v[j].t0, v[j].n, 0, 0, 0};
    group[j] = g;
  }
  __syncthreads();
  // Every group for both numbers of row tiles, as long as the mean is not known: members[g] becomes the bits of those with which it shares
  for (u32 g = threadIdx.x; g < a.n_groups; g += NT) {
    u32 shares = 0, which = 0;
    // (cu_seqlens that decrease may have the first member's tokens behind another one's, or a token in two members: then the rows from t0 on would not hold them, and there is no group)
    if (members[g] > 1 && view[from[g]].t0 == t0[g] && queries[g] <= t1[g] - t0[g]) {
      const u32 n = queries[g], tiles = keys[g] / 16;
      const bool apart = n < t1[g] - t0[g];
      if (BY_MEAN) atomicAdd(sizes + g % SPREAD, GROUPS_UNIT + n);
      for (u32 o = 0; o < OPTIONS; ++o) {
        const u32 rows = BY_MEAN ? (o ? a.most_rows : 16u) : a.short_rows;
        const float few_cost = a.few_cost * (rows > 16 ? FEW_MORE : 1.f);
        const float together = n * a.G <= rows && !apart ? few_cost * (float)(tiles + FEW_PAIR) : (float)flat_shape(a, n * a.G, keys[g]).all();
        const float gain = (float)members[g] * (float)tiles * few_cost - together - a.row_cost * (float)n;
        if (!a.share_all && !(gain > SHARED_GAIN)) continue;
        shares |= 1u << o;
        if (!a.share_all) atomicAdd(gained + o * SPREAD + g % SPREAD, (u32)min(gain, 1e6f));      // (1024 times that is less than 2^32)
      }
      which = from[g] + (apart ? PAGED_MAX_SEQS : 0u);
      if (apart && shares) *gaps = 1;
    }
    members[g] = shares;
    view[a.n_seqs + g] = SharedView{t0[g], queries[g], (i32)keys[g] - 1, 0, which};
  }
  __syncthreads();
  u32 option = 0, all_gained = 0;
  if (BY_MEAN) {
    u32 all = 0;
    for (u32 i = 0; i < SPREAD; ++i) all += sizes[i];
    const u32 n = all / GROUPS_UNIT, mean = n ? (all % GROUPS_UNIT + n - 1) / n : 0u;
    option = (*some_rows && !*many_rows) || (mean * a.G > 16 && mean * a.G <= a.most_rows) ? 1 : 0;
    a.short_rows = option ? a.most_rows : 16u;
  }
  for (u32 i = 0; i < SPREAD; ++i) all_gained += gained[option * SPREAD + i];
  const bool share = a.share_all || all_gained >= a.gain;
  for (u32 g = threadIdx.x; g < a.n_groups; g += NT) if (!share || !(members[g] >> option & 1u)) view[a.n_seqs + g] = SharedView{0, 0, -1, 0, 0};
  u32 before[EACH] = {};
  if (share && *gaps) {                              // members' queries before every sequence: sums over 1, 2, 4 .. sequences
    u32 *sum = scratch, *next = sum + PAGED_MAX_SEQS;
#pragma unroll
    for (u32 j = 0; j < EACH; ++j)
      if (threadIdx.x + j * NT < a.n_seqs) sum[threadIdx.x + j * NT] = group[j] == NO_GROUP ? 0u : v[j].n;
    __syncthreads();
    for (u32 step = 1; step < a.n_seqs; step *= 2) {
      for (u32 s = threadIdx.x; s < a.n_seqs; s += NT) next[s] = sum[s] + (s >= step ? sum[s - step] : 0u);
      __syncthreads();
      u32* const x = sum;
      sum = next; next = x;
    }
#pragma unroll
    for (u32 j = 0; j < EACH; ++j) {
      const u32 s = threadIdx.x + j * NT;
      if (s && s < a.n_seqs) before[j] = sum[s - 1];
    }
  }
#pragma unroll
  for (u32 j = 0; j < EACH; ++j) {
    const u32 s = threadIdx.x + j * NT, g = group[j];
    if (s >= a.n_seqs) continue;
    const bool in = share && g != NO_GROUP && (members[g] >> option & 1u);
    view[s] = SharedView{v[j].t0, v[j].n, v[j].pos0, in ? keys[g] : 0u, (in ? g : 0u) + PAGED_MAX_SEQS * before[j]};
  }
  __syncthreads();
}

// token of query k of a group, and which of a group's queries is query k of a sequence of its
__device__ __forceinline__ u32 group_token(const SharedArgs& a, const SharedView* view, const SharedView& group, u32 k) {
  if (!group.gaps()) return group.t0 + k;
  u32 s = group.row();                               // the last sequence with so many of the group's queries before it, or fewer
  const u32 base = view[s].before();
  for (u32 step = PAGED_MAX_SEQS / 2; step; step >>= 1) if (s + step < a.n_seqs && view[s + step].before() - base <= k) s += step;
  return view[s].t0 + k - (view[s].before() - base);
}
__device__ __forceinline__ u32 member_query(const SharedArgs& a, const SharedView* view, const SharedView& group, const SharedView& v, u32 k) {
  return k + (group.gaps() ? v.before() - view[group.row()].before() : v.t0 - group.t0);
}
// The row of results to be joined, of every query head, for query k of a sequence whose first token is t0 (a group: its first member's; its members have as many rows as it has queries). A sequence
// of SHARED_ROWS rows or more, a prompt, has none: what a call needs room for does not grow with its prompts.
__host__ inline void rows_of_call(SharedArgs& a) {
  const u32 most = (SHARED_ROWS - 1) / a.G, each = a.max_q < most ? a.max_q : most;
  a.row_tokens = (u64)a.n_seqs * each < a.n_tokens ? each : 0;
  a.n_rows = a.row_tokens ? a.n_seqs * each : a.n_tokens;
}
__device__ __forceinline__ u32 row_index(const SharedArgs& a, u32 s, u32 t0, u32 k) { return (a.row_tokens ? s * a.row_tokens : t0) + k; }

__device__ __forceinline__ u32 short_unit_count(const PagedArgs& a, const SeqView& v) {     // tiles of a sequence and kv head; 0: not this part's, 1 at least else
  if (!v.n || v.n * a.G > a.short_rows) return 0;
  return max(1u, seen_tiles<16>(a, v.pos0, v.pos0 + (i32)v.n - 1).n);
}
__device__ __forceinline__ u32 short_unit_count(const SharedArgs& a, const SharedView& v, bool group) {
  if (!v.n || v.n * a.G > a.short_rows || (group && v.gaps())) return 0;
  return max(1u, seen_tiles<16>(a, v.pos0, group ? v.pos0 : v.pos0 + (i32)v.n - 1, v.first).n);
}
template <typename View>
__device__ __forceinline__ u32 prompt_items(const PagedArgs& a, const View& v) {
  return v.n * a.G <= a.short_rows ? 0u : (v.n * a.G + PROMPT_ROWS - 1) / PROMPT_ROWS;
}
// parts of every item's keys: as many as there are workgroups for
__device__ __forceinline__ u32 prompt_parts(const PagedArgs& a, u32 items, u32 nwg) { return items && items < nwg ? max(1u, min(a.n_splits, nwg / items)) : 1u; }

struct PromptItem { u32 s, g, r0, rows, t0; i32 p0, p1; u32 lo, row; };      // rows r0 .. r0 + rows of the view's, queries at positions p0 .. p1; first key, row of the table
struct FlatRun { u32 from, end; };
struct FlatPiece { u32 s_lo, s_hi, next; bool whole, begins, any; };       // any: has units of steps (of steps themselves perhaps none)
// the slot of workgroup wg's result of an item that other runs have as well, by whether the item begins in its run
__device__ __forceinline__ u32 flat_slot(u32 wg, bool begins) { return 2 * wg + (begins ? 1u : 0u); }
// what a run that ends at `end` has from unit u on, of the item that u is in: of group g, whose units begin at unit `first`
__device__ __forceinline__ PromptItem flat_piece(const SharedArgs& a, const SharedView& v, u32 g, u32 first, u32 u, u32 end, FlatPiece& p) {
  PromptItem it;
  const FlatShape f = flat_shape(a, v);
  const u32 all = f.all(), x = u - first, head = x / all, full = FLAT_STEP * f.steps + f.lead, item = min((x - head * all) / full, f.items - 1);
  const u32 per = f.units(item), off = x - head * all - item * full, to = min(per, off + end - u), weight = item + 1 < f.items ? FLAT_STEP : f.last;
  auto step = [&](u32 at) { return at > f.lead ? (at - f.lead + weight - 1) / weight : 0u; };
  p = {step(off), step(to), u + to - off, off <= f.lead && to == per, off <= f.lead, to > f.lead};
  it.s = a.n_seqs + g;
  it.g = head;
  it.r0 = item * flat_rows(a);
  it.rows = min(flat_rows(a), v.n * a.G - it.r0);
  it.t0 = v.t0; it.p0 = it.p1 = v.pos0; it.lo = 0; it.row = v.row();
  return it;
}

// What a view adds to the sums: prompt items, units of the groups' shared keys, tiles of few rows (times kv heads), units of the prompt items' steps
__device__ __forceinline__ void view_units(const SharedArgs& a, const SharedView& x, bool group, u32 (&v)[4]) {
  if (group) v[1] = flat_units(a, x); else v[0] = prompt_items(a, x);
  const u32 tiles = short_unit_count(a, x, group);
  v[2] = (tiles ? tiles + FEW_PAIR : 0u) * a.nkv;
  // (a time to go by, and that there is some: an item's, in the middle between the first one's and the last one's, held to a second's, so that 1024 of them stay within 32 bits)
  if (v[0]) {
    const i32 p1 = x.pos0 + (i32)x.n - 1, some = (i32)min(x.n, PROMPT_ROWS / a.G) - 1;
    const u32 steps = seen_tiles<64>(a, x.pos0, x.pos0 + some, x.first).n + seen_tiles<64>(a, p1 - some, p1, x.first).n;
    v[3] = (u32)min((u64)v[0] * (FLAT_STEP * steps / 2 + a.lead) * a.nkv, (u64)1 << 21);
  }
}

// The work of a call with groups, by every workgroup all the same: views, who has the groups' shared keys and who the rest. Then notes for the join.
struct SharedWork { u32 flat_wgs, quota; bool few, prompts; };
// Workgroups for the groups' shared keys and for the rest, by their estimated times, and the units of a run of the former. Where there are prompts, whose items come from a counter, the former
// take some of them at their runs' end, so one too many loses nothing
__device__ __forceinline__ SharedWork deal_out(const SharedArgs& a, u32 units, u32 tiles, u32 prompts, u32 nwg) {
  SharedWork r;
  r.few = tiles != 0; r.prompts = prompts != 0;
  const float flat = (float)units, rest = a.few_cost * (a.short_rows > 16 ? FEW_MORE : 1.f) * (float)tiles + (float)prompts;
  r.flat_wgs = !units ? 0u : rest == 0.f ? nwg : min(nwg - 1, max(1u, (u32)((float)nwg * flat / (flat + rest) + (prompts ? 1.f : 0.5f))));
  r.quota = r.flat_wgs ? (units + r.flat_wgs - 1) / r.flat_wgs : 1u;
  return r;
}
// What is to be joined of a token's rows (kinds 0: nothing, its results are in place; 1: a result of its group and one of its sequence; 2: parts of a prompt
// item's keys). Its group's: units[0] + kv head * units[1] is where its item's line of units[2] begins, row: its first row there. Its sequence's:
// in rows, or parts of prompt items (parts > 1): items top - (row + head) / PROMPT_ROWS. rows: of the group's result and the sequence's, where those are in rows.
struct alignas(16) JoinToken { u32 kind : 2, row : 9, parts : 21, units[3], own_row, top, rows[2]; };
// Of token t: the views, items of the prompts before each sequence (pre), units before each group (flat), parts of every prompt item
__device__ __forceinline__ JoinToken join_token(const SharedArgs& a, const SharedView* view, const u32* pre, const u32* flat, u32 parts, u32 t) {
  u32 s = 0;                                       // the last sequence that begins at this token or before
  for (u32 step = PAGED_MAX_SEQS / 2; step; step >>= 1) if (s + step < a.n_seqs && view[s + step].t0 <= t) s += step;
  const SharedView v = view[s];
  JoinToken j = {};
  if (t >= v.t0 && t - v.t0 < v.n) {
    const bool cut = parts > 1 && prompt_items(a, v) != 0;
    j.own_row = (t - v.t0) * a.G; j.top = pre[a.n_seqs] - 1 - pre[s]; j.parts = cut ? parts : 1;
    j.kind = v.first ? 1 : cut ? 2 : 0;
    j.rows[1] = row_index(a, s, v.t0, t - v.t0);
    if (v.first) {
      const SharedView x = view[a.n_seqs + v.group()];
      const u32 k = member_query(a, view, x, v, t - v.t0), r = k * a.G;
      j.rows[0] = row_index(a, x.row(), x.t0, k);
      if (flat_units(a, x)) {
        const FlatShape f = flat_shape(a, x);
        const u32 item = r / flat_rows(a);
        j.units[0] = flat[v.group()] + item * (FLAT_STEP * f.steps + f.lead) + f.lead; j.units[1] = f.all(); j.units[2] = f.units(item) - f.lead;
        j.row = r - item * flat_rows(a);
      } else j.units[2] = 1;                       // (by one workgroup, into rows)
    }
  }
  return j;
}

// Times on one compute unit, by which workgroups are dealt out. A unit: a quarter of a step of 256 rows, see FlatShape. Against units of half a step, with one for a step of 128 rows or less
// (two over 4 bits): up to 96 sequences with 5 drafts 82 us, so 76 in 4 bits, 82 and 73 over halves; 12 groups of 70 120, 107; 200 sequences of heads of 64 71, 60; three groups of 30 52, 53.
// 16 groups of 8 sequences, 32 rows each, 59, and with FLAT_LIGHT for them 63
__host__ inline void shared_costs(SharedArgs& p, u32 hd, u32 bits, u32 n_cu) {
  const bool halves = bits == 16;
  const float unit = hd == 128 ? (halves ? 0.47f : 0.56f) : (halves ? 0.38f : 0.49f);
  p.lead = hd == 128 ? 13 : halves ? 18 : 9;
  p.least = halves ? 2 : FLAT_LIGHT;
  p.most_rows = 16 * SHORT_MORE(hd);
  const u64 own = (u64)p.max_q * p.G, all = (u64)p.n_tokens * p.G;
  p.short_rows = (all <= p.most_rows ? all > 16 : own > 16 && own <= p.most_rows) ? p.most_rows : 16u;
  p.few_cost = halves ? 0.6f : 0.26f;
  // (what sharing must gain on every compute unit: 8 us for the groups' starts and the join, and what the members' rows take to memory and back: of other tokens nothing is joined. Shared and apart in us: 64 sequences in
  // 4 bits, 1024 shared keys: 30, 28; 253 behind 64: 70, 61; 16 groups of 8 behind 64: 35, 37; 40 groups of 4, heads of 64, behind 64: 26, 25)
  const float units = (float)n_cu / (float)p.nkv / unit;      // of a us, for a kv head
  p.gain = (u32)(8.f * units);
  p.row_cost = (float)p.nq * (float)(16 * ROW_RESULT(hd)) * 2e-7f * units;
}
