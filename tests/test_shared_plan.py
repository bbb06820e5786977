"""Who has which part of a call with groups, gone through on the CPU: views, units, runs, slots and rows of the workspace, and what the join reads of them (no GPU needed)."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_07609_amd", "csrc")

# The header as one thread, and everything that a call's workgroups do with it: pieces of the groups' shared keys with their slots, rows written, then
# the join of every row. go_through returns 0, or the line of the first rule that is broken.
HARNESS = r"""
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstdlib>
#include <map>
#include <vector>
typedef uint32_t u32;
typedef uint64_t u64;
typedef int32_t i32;
typedef uint16_t f16_t;
#define __device__
#define __host__
#define __forceinline__ inline
static struct { u32 x; } threadIdx;
static void __syncthreads() {}
static int __clz(int x) { return __builtin_clz((unsigned)x); }
static u32 atomicAdd(u32* p, u32 v) { const u32 o = *p; *p += v; return o; }
static u32 atomicMin(u32* p, u32 v) { const u32 o = *p; *p = std::min(o, v); return o; }
static u32 atomicMax(u32* p, u32 v) { const u32 o = *p; *p = std::max(o, v); return o; }
static u32 atomicOr(u32* p, u32 v) { const u32 o = *p; *p |= v; return o; }
using std::max;
using std::min;
#include "paged_views.h"
#define RULE(x) do { if (!(x)) return __LINE__; } while (0)

struct Call { u32 nq, nkv, hd, bits, n_seqs, n_tokens, max_q, max_blocks, window, sinks, n_groups, share_all, nwg, n_splits; const i32 *cu, *lens, *starts, *shared; };
// of every sequence: first key of its own; of every group: queries; then workgroups of the shared keys, rows of few, units, tiles, prompts' units
extern "C" int go_through(const Call* c, u32* first, u32* queries, u32* of_call) {
  SharedArgs a{};
  a.nq = c->nq; a.nkv = c->nkv; a.G = c->nq / c->nkv; a.n_seqs = c->n_seqs; a.n_tokens = c->n_tokens; a.max_q = c->max_q; a.max_blocks = c->max_blocks;
  a.window = c->window; a.sinks = c->sinks; a.n_groups = c->n_groups; a.share_all = c->share_all; a.n_splits = c->n_splits;
  a.cu = c->cu; a.lens = c->lens; a.starts = c->starts; a.shared = c->shared;
  shared_costs(a, c->hd, c->bits, c->nwg);
  rows_of_call(a);
  RULE(a.n_rows <= a.n_tokens);
  std::vector<u32> room(ROOM_WORDS), pre(PAGED_MAX_SEQS + 1), flat(PAGED_MAX_SEQS + 1);
  std::vector<SharedView> view(PAGED_MAX_SEQS);
  if (rows_by_mean(c->hd, c->bits)) shared_views<1, true>(a, room.data(), view.data());
  else shared_views<1, false>(a, room.data(), view.data());
  u64 sums[4] = {0, 0, 0, 0}, all_units = 0;
  for (u32 s = 0; s < n_views(a); ++s) {
    u32 v[4] = {0, 0, 0, 0};
    view_units(a, view[s], s >= a.n_seqs, v);
    for (int k = 0; k < 4; ++k) sums[k] += v[k];
    if (s < a.n_seqs) pre[s + 1] = (u32)sums[0]; else flat[s - a.n_seqs + 1] = (u32)sums[1];
    if (s >= a.n_seqs && v[1]) {
      const FlatShape f = flat_shape(a, view[s]);
      all_units += (((u64)f.items - 1) * ((u64)FLAT_STEP * f.steps + f.lead) + (u64)f.last * f.steps + f.lead) * a.nkv;
    }
  }
  for (int k = 0; k < 4; ++k) RULE(sums[k] < 1ull << 32);
  RULE(sums[1] == all_units && all_units + c->nwg < 1ull << 32);
  const SharedWork w = deal_out(a, (u32)sums[1], (u32)sums[2], (u32)sums[3], c->nwg);
  RULE(w.flat_wgs <= c->nwg && (w.flat_wgs < c->nwg || !(w.few || w.prompts)) && (w.flat_wgs > 0) == (sums[1] > 0));
  RULE((u64)w.quota * std::max(w.flat_wgs, 1u) >= sums[1]);
  // (beside prompts, whose items whoever is free takes, no run of the shared keys is longer than everyone's share of all the work)
  const double rest = a.few_cost * (a.short_rows > 16 ? FEW_MORE : 1.f) * (double)sums[2] + (double)sums[3];
  RULE(!w.flat_wgs || !w.prompts || w.flat_wgs == c->nwg - 1 || (double)sums[1] / w.flat_wgs <= 1.001 * (sums[1] + rest) / c->nwg);
  const u32 items = pre[a.n_seqs] * a.nkv, parts = prompt_parts(a, items, c->nwg - w.flat_wgs);
  RULE(parts == 1 || (u64)items * parts <= c->nwg);
  for (u32 s = 0; s < a.n_seqs; ++s) first[s] = view[s].first;
  for (u32 g = 0; g < a.n_groups; ++g) queries[g] = view[a.n_seqs + g].n;
  of_call[0] = w.flat_wgs; of_call[1] = a.short_rows; of_call[2] = (u32)sums[1]; of_call[3] = (u32)sums[2]; of_call[4] = (u32)sums[3];

  bool ascending = true, groups_ascending = true;
  for (u32 s = 0; s < a.n_seqs; ++s) ascending &= a.cu[s] >= 0 && a.cu[s] <= a.cu[s + 1];
  for (u32 g = 0; g < a.n_groups; ++g) groups_ascending &= a.starts[g] <= a.starts[g + 1];
  const bool ordered = ascending && groups_ascending;

  // what is written: rows by (which, row, kv head) -> (view, query); slots -> (group, kv head, first row)
  struct Written { u32 view, query; };
  std::map<std::vector<u32>, Written> rows;
  struct Slot { u32 g, head, r0, rows, s_lo, s_hi; bool used; };
  std::vector<Slot> slots(2 * c->nwg, Slot{});
  auto wrote = [&](u32 which, const SharedView& v, u32 index, u32 query, u32 head) {
    const u32 row = row_index(a, which ? index : v.row(), v.t0, query);
    if (row >= a.n_rows) return false;
    // (two views' rows at the same place only where what comes out is not defined)
    if (ordered && rows.count({which, row, head})) return false;
    rows[{which, row, head}] = {index, query};
    return true;
  };
  for (u32 g = 0; g < a.n_groups; ++g) {
    const SharedView& v = view[a.n_seqs + g];
    for (u32 k = 0; k < v.n; ++k) RULE(group_token(a, view.data(), v, k) < a.n_tokens);
    if (v.n && !flat_units(a, v))
      for (u32 k = 0; k < v.n; ++k) for (u32 h = 0; h < a.nkv; ++h) RULE(wrote(0, v, a.n_seqs + g, k, h));
  }
  for (u32 x = 0; x < w.flat_wgs; ++x) {
    const u32 from = (u32)std::min<u64>((u64)x * w.quota, sums[1]), end = (u32)std::min<u64>((u64)from + w.quota, sums[1]);
    for (u32 u = from; u < end;) {
      u32 g = 0;
      while (g + 1 < a.n_groups && flat[g + 1] <= u) ++g;
      const SharedView& v = view[a.n_seqs + g];
      FlatPiece p;
      const PromptItem it = flat_piece(a, v, g, flat[g], u, end, p);
      if (!p.any) { RULE(p.next == end); break; }
      RULE(it.g < a.nkv && it.rows && it.rows <= PROMPT_ROWS && it.r0 % a.G == 0 && (u64)it.r0 + it.rows <= (u64)v.n * a.G);
      RULE(p.s_lo <= p.s_hi && p.s_hi <= (u32)(v.pos0 + 1) / 64 && p.next > u && p.next <= end && it.row < a.n_seqs);
      if (p.whole) {
        RULE(p.s_lo == 0 && p.s_hi == (u32)(v.pos0 + 1) / 64);
        for (u32 r = 0; r < it.rows; r += a.G) RULE(wrote(0, v, a.n_seqs + g, (it.r0 + r) / a.G, it.g));
      } else {
        Slot& s = slots[flat_slot(x, p.begins)];
        RULE(!s.used);
        s = {g, it.g, it.r0, it.rows, p.s_lo, p.s_hi, true};
      }
      u = p.next;
    }
  }
  for (u32 s = 0; s < a.n_seqs; ++s) {
    const SharedView& v = view[s];
    if (v.first && !(parts > 1 && prompt_items(a, v)))
      for (u32 k = 0; k < v.n; ++k) for (u32 h = 0; h < a.nkv; ++h) RULE(wrote(1, v, s, k, h));
  }
  // the join (groups that decrease may have sequences between one another's, cu_seqlens that do may have a token in two sequences: what comes out is not defined then, and
  // only where it is written and read is looked at)
  std::vector<u32> joined(a.n_seqs);
  for (u32 t = 0; t < a.n_tokens; ++t) {
    const JoinToken j = join_token(a, view.data(), pre.data(), flat.data(), parts, t);
    if (!j.kind) continue;
    u32 s = 0;
    while (s < a.n_seqs && !(view[s].t0 <= t && t - view[s].t0 < view[s].n)) ++s;
    RULE(s < a.n_seqs);
    const bool one = ordered;
    ++joined[s];
    const SharedView& v = view[s];
    const u32 query = t - v.t0;
    for (u32 h = 0; h < a.nkv; ++h) {
      auto row = [&](u32 which, u32 index, u32 q) {
        RULE(j.rows[which] < a.n_rows);
        const auto found = rows.find({which, j.rows[which], h});
        if (!one) return 0;
        RULE(found != rows.end() && found->second.view == index && found->second.query == q);
        return 0;
      };
      if (j.kind == 1) {
        const u64 begin = (u64)j.units[0] + (u64)h * j.units[1];
        RULE(begin + j.units[2] <= std::max<u64>(sums[1], 1));
        const u32 w0 = (u32)(begin / w.quota), w1 = (u32)((begin + j.units[2] - 1) / w.quota);
        const u32 g = view[s].group(), k = member_query(a, view.data(), view[a.n_seqs + g], v, query);
        if (w0 == w1) { if (int rc = row(0, a.n_seqs + g, k)) return rc; }
        else {
          RULE(w1 < w.flat_wgs && j.row + a.G <= PROMPT_ROWS);
          u32 steps = 0;
          for (u32 x = w0; x <= w1; ++x) {
            const Slot& q = slots[flat_slot(x, x == w0)];
            if (!one) continue;
            RULE(q.used && q.g == g && q.head == h && q.r0 + j.row == k * a.G && j.row < q.rows && q.s_lo == steps);
            steps = q.s_hi;
          }
          RULE(!one || steps == (u32)(view[a.n_seqs + g].pos0 + 1) / 64);
        }
      }
      if (j.parts > 1) {
        for (u32 i = 0; i < a.G; ++i) {
          const u32 r = j.own_row + i, item = (j.top - r / PROMPT_ROWS) * a.nkv + h;
          RULE(j.top >= r / PROMPT_ROWS && (u64)(item + 1) * j.parts <= c->nwg);
        }
      } else if (int rc = row(1, s, query)) return rc;
    }
  }
  for (u32 s = 0; s < a.n_seqs && ascending; ++s)
    RULE(joined[s] == (view[s].first || (parts > 1 && prompt_items(a, view[s])) ? view[s].n : 0u));
  return 0;
}
"""
class Call(ctypes.Structure):
    _fields_ = [(n, ctypes.c_uint32) for n in ("nq", "nkv", "hd", "bits", "n_seqs", "n_tokens", "max_q", "max_blocks", "window", "sinks", "n_groups", "share_all", "nwg", "n_splits")] + [
        (n, ctypes.c_void_p) for n in ("cu", "lens", "starts", "shared")]


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("shared")
    (tmp / "plan.cpp").write_text(HARNESS)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wno-unknown-pragmas", "-shared", "-fPIC", "-I", CSRC, "-o", str(tmp / "plan.so"), str(tmp / "plan.cpp")], check=True)
    lib = ctypes.CDLL(str(tmp / "plan.so"))

    def run(cu, lens, starts, shared, nq=32, nkv=8, hd=128, bits=16, window=0, sinks=0, share_all=1, nwg=256, max_q=None, n_tokens=None, max_blocks=None):
        """(first key of every sequence's own, queries of every group, [workgroups of the shared keys, rows of few, units, tiles, prompts' units])"""
        cu, lens, starts, shared = (np.int32(x) for x in (cu, lens, starts, shared))
        max_blocks = max_blocks or max(1, (int(max(lens)) + 15) // 16)
        max_q = max_q or max(1, int(np.diff(cu).max()))
        T = n_tokens or int(max(cu))
        c = Call(nq, nkv, hd, bits, len(lens), T, max_q, max_blocks, window, sinks, len(shared), share_all, nwg, max(1, (max_blocks // 4 + 1) // 4),
                 *(x.ctypes.data for x in (cu, lens, starts, shared)))
        first, queries, of_call = np.zeros(len(lens), np.uint32), np.zeros(len(shared) + 1, np.uint32), np.zeros(8, np.uint32)
        line = lib.go_through(ctypes.byref(c), *(x.ctypes.data_as(ctypes.c_void_p) for x in (first, queries, of_call)))
        assert line == 0, HARNESS.split("\n")[line - 1]
        return first.tolist(), queries[:-1].tolist(), of_call.tolist()

    return run


def batch(seqs):
    """[(context, queries, group or None) ...], sequences of a group together -> cu, lens, starts of the groups"""
    cu = np.concatenate(([0], np.cumsum([m for _, m, _ in seqs])))
    groups = sorted({g for _, _, g in seqs if g is not None})
    starts = [min(i for i, s in enumerate(seqs) if s[2] == g) for g in groups]
    return cu, [n for n, _, _ in seqs], starts + [max(i for i, s in enumerate(seqs) if s[2] == groups[-1]) + 1]


HEADS = [(32, 8, 128, 16), (32, 4, 128, 4), (16, 16, 64, 16), (33, 1, 64, 4), (64, 1, 128, 16)]


@pytest.mark.parametrize("share_all", [0, 1])
@pytest.mark.parametrize("nwg", [256, 64])
@pytest.mark.parametrize("nq, nkv, hd, bits", HEADS)
def test_every_row_is_written_where_the_join_reads_it(plan, nq, nkv, hd, bits, nwg, share_all):
    for seed in range(40):
        rng = np.random.default_rng(seed)
        n_groups = int(rng.integers(1, 9))
        seqs, shared = [], []
        for g in range(n_groups):
            sh = int(np.exp(rng.uniform(0, 9.5)))
            shared.append(sh)
            for _ in range(int(np.exp(rng.uniform(0, 4)))):
                m = int(rng.choice([0, 1, 1, 1, 2, 5, 9, 17, 40, 70, 300], p=[.05, .3, .15, .1, .1, .1, .05, .05, .04, .03, .03]))
                seqs.append((max(0, sh + m + int(rng.choice([-40, 0, 3, 100, 1000]))), m, g))
            if rng.random() < 0.3:
                seqs.append((int(rng.integers(1, 3000)), int(rng.choice([1, 5, 200])), None))
        if seqs[-1][2] is None:
            seqs.pop()
        if len(seqs) + n_groups > 1024 or not any(m for _, m, _ in seqs):
            continue
        # (a sequence in no group behind its predecessor's: in that one's range of sequences, with blocks that need not agree)
        plan(*batch(seqs), shared, nq, nkv, hd, bits, nwg=nwg, share_all=share_all, window=int(rng.choice([0, 0, 0, 500])))


@pytest.mark.parametrize("nq, nkv, hd, bits", HEADS)
def test_lengths_groups_and_tokens_that_do_not_fit(plan, nq, nkv, hd, bits):
    """Numbers that come from device memory may be anything: nothing is read or written outside of the call's tensors then."""
    for seed in range(300):
        rng = np.random.default_rng(1000 + seed)
        S, G = int(rng.integers(1, 60)), int(rng.integers(1, 6))
        any_ = lambda n, lo, hi: np.where(rng.random(n) < 0.1, rng.choice([-2 ** 31, -1, 2 ** 31 - 1], n), rng.integers(lo, hi, n))      # noqa: E731
        cu = np.where(rng.random(S + 1) < 0.7, np.sort(rng.integers(0, 200, S + 1)), any_(S + 1, 0, 200))
        plan(cu, any_(S, 0, 3000), any_(G + 1, 0, S + 1), any_(G, 0, 1500), nq, nkv, hd, bits, max_q=int(rng.integers(1, 90)), n_tokens=200, max_blocks=190)


# cu_seqlens that decrease between members of one group of (context, queries) behind 128 shared tokens; the queries of the group that is formed all the same (0: none is)
DECREASING = [
    ([4, 6, 9, 5, 7], [140, 141, 130, 139], 0),                          # more queries than tokens between the first and the last one
    ([0, 2, 20, 22, 10, 12], [140, 100, 135, 130, 200], 6),              # one that may not share between them, then an unused one
    ([0, 1, 3, 5, 3, 5], [140, 100, 135, 130, 200], 5),                  # two members with the same tokens
    ([10, 12, 2, 4, 6], [140, 130, 150, 160], 0),                        # the first member's tokens behind the others'
]


@pytest.mark.parametrize("cu, lens, queries", DECREASING)
@pytest.mark.parametrize("times", [1, 30])
@pytest.mark.parametrize("nq, nkv, hd, bits", HEADS)
def test_decreasing_tokens_inside_a_group(plan, nq, nkv, hd, bits, times, cu, lens, queries):
    """Alone and as one of many members, the others ahead of it."""
    more = 2 * (times - 1)
    cu = [2 * i for i in range(times - 1)] + [more + x for x in cu]
    got = plan(cu, [140] * (times - 1) + lens, [0, len(cu) - 1], [128], nq, nkv, hd, bits, n_tokens=max(cu) + 2, max_blocks=16)[1]
    if times == 1:
        assert got == [queries]


@pytest.mark.parametrize("share_all", [0, 1])
@pytest.mark.parametrize("nq, nkv, hd, bits", HEADS)
@pytest.mark.parametrize("members, queries", [(24, 1), (64, 1), (150, 1), (30, 3)])
def test_a_sequence_that_may_not_share_takes_nothing_from_its_neighbours(plan, nq, nkv, hd, bits, members, queries, share_all):
    """A chunk of a prompt, and a sequence whose context lies within the shared tokens: the group is the same wherever in its range they stand."""
    shared, group = 6000, [(6000 + queries + 7 * i, queries, 0) for i in range(members)]
    alien = [(9000, 3000, 0), (500, 2, 0)]
    behind = plan(*batch(group + alien), [shared], nq, nkv, hd, bits, share_all=share_all)
    keys = behind[0][0]                                # (0 with one kv head and few members: too little work to gain by)
    assert behind[1] == [members * queries if keys else 0] and behind[0] == [keys] * members + [0, 0]
    assert keys == shared // 64 * 64 or (nkv == 1 and not share_all)
    for at in (0, 1, members // 2, members - 1):
        first, n, of_call = plan(*batch(group[:at] + alien + group[at:]), [shared], nq, nkv, hd, bits, share_all=share_all)
        assert n == behind[1] and first == [keys] * at + [0, 0] + [keys] * (members - at), at


@pytest.mark.parametrize("nq, nkv, hd, bits", HEADS)
@pytest.mark.parametrize("context, queries", [(2000, 2000), (9000, 4000), (8192, 8192), (40000, 512)])
def test_prompts_beside_groups(plan, nq, nkv, hd, bits, context, queries):
    """Units of a prompt's items: those of the steps that each of them has, not of the longest one's; and no long run of shared keys beside it (a rule of the harness)."""
    G = nq // nkv
    of_call = plan(*batch([(4100 + i, 1, 0) for i in range(32)] + [(context, queries, None)]), [4000], nq, nkv, hd, bits)[2]
    rows = [min(256, queries * G - r) + r for r in range(0, queries * G, 256)]
    steps = [(context - queries + (r - 1) // G) // 64 + 1 for r in rows]
    want = sum(4 * s + 13 for s in steps) * nkv
    assert want < 2 ** 21 and abs(of_call[4] - want) < 0.05 * want + 6 * len(steps) * nkv


@pytest.mark.parametrize("nq, nkv, hd, bits", HEADS)
@pytest.mark.parametrize("members, shared", [(2, 70), (4, 1040), (16, 8000), (32, 4000), (64, 2000), (100, 300), (200, 64), (12, 500)])
def test_whether_groups_share_does_not_depend_on_who_is_beside_them(plan, nq, nkv, hd, bits, members, shared):
    """Prompts and sequences in no group are not joined, so they change nothing of what sharing gains."""
    group = [(shared + 1 + i, 1, 0) for i in range(members)]
    alone = plan(*batch(group), [shared], nq, nkv, hd, bits, share_all=0)
    for beside in ([(2000, 2000, None)], [(8192, 8192, None)], [(1000 + i, 1, None) for i in range(100)]):
        assert plan(*batch(group + beside), [shared], nq, nkv, hd, bits, share_all=0)[1] == alone[1]


@pytest.mark.parametrize("nq, nkv, hd, bits, groups, members, queries, rows", [
    (32, 8, 128, 4, 16, 8, 1, 32), (32, 8, 128, 4, 16, 9, 1, 16), (32, 8, 128, 4, 5, 4, 1, 16), (16, 16, 64, 16, 40, 4, 9, 64), (32, 8, 64, 4, 3, 16, 1, 64),
    (32, 8, 64, 16, 3, 17, 1, 16), (16, 16, 64, 16, 30, 2, 8, 16), (32, 8, 128, 16, 16, 8, 1, 16)])
def test_row_tiles_are_those_that_the_groups_need(plan, nq, nkv, hd, bits, groups, members, queries, rows):
    """Rows of the few-row part: by the mean of the groups there are, whoever is beside them; then by sequences that need more than 16, unless some need more than it holds."""
    seqs, shared = [(1500 + queries + i, queries, g) for g in range(groups) for i in range(members)], [1500] * groups
    assert plan(*batch(seqs), shared, nq, nkv, hd, bits)[2][1] == rows
    for beside in ([(1000 + i, 1, None) for i in range(100)], [(2000, 2000, None)]):
        assert plan(*batch(seqs + beside), shared, nq, nkv, hd, bits)[2][1] == rows
    few = [(300, 24 * nkv // nq, None)]                  # 24 rows
    assert plan(*batch(seqs + few), shared, nq, nkv, hd, bits)[2][1] == (32 if hd == 128 else 64)
    assert plan(*batch(seqs + few + [(2000, 2000, None)]), shared, nq, nkv, hd, bits)[2][1] == rows


def test_units_at_the_largest_sizes(plan):
    """A chunk of 131072 queries among 4 M shared tokens between two members, 8 kv heads: with its rows the units would not fit 32 bits. Then as many members as there may be."""
    long = 1 << 22
    assert plan(*batch([(long + 1, 1, 0), (long, 131072, 0), (long + 5, 1, 0)]), [long])[1] == [2]
    members = [(4 * 64 + 63, 63, 0)] * 1000
    assert plan(*batch(members), [4 * 64], nq=32, nkv=8, max_blocks=260000)[1] == [63000]
    deep = (1 << 31) // (1001 * 8) - 1                   # blocks of each
    assert plan(*batch([(deep * 16 - 1, 7, 0)] * 1000), [deep * 16 - 64], nq=264, nkv=8, max_blocks=deep)[1] == [7000]
