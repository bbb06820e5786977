"""Attention of groups in batches that hold other sequences as well: between the members of a group, beside the groups, and with lengths that do not fit."""
import numpy as np
import pytest
import torch

import paper_2604_07609_amd as B
from tests.test_gpu_operators import check_attention, dev, no_error_of_earlier_tests  # noqa: F401
from tests.test_gpu_operators_shared import check, make_groups, run_shared
from tests.test_shared_plan import DECREASING

pytestmark = pytest.mark.gpu

HEADS = [(64, 6, 2), (128, 4, 1), (64, 33, 1)]


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("hd, nq, nkv", HEADS)
@pytest.mark.parametrize("groups", [
    [(130, [(140, 1), (500, 300), (141, 4)])],                                           # a prompt between the only two members
    [(130, [(500, 300), (140, 2), (100, 30), (150, 1), (20, 20), (135, 3), (430, 280)])],
    [(200, [(201 + i, 1) if i % 7 else (400, 270 if i % 2 else 150) for i in range(1, 40)])],      # many, with some that have many queries
    [(128, [(129 + i, 1 + i % 3) for i in range(25)] + [(90, 2)] + [(140, 12)] * 9), (70, [(75, 1), (60, 1), (90, 5)])],
    [(64, [(70, 1), (66, 3), (20, 1)]), (0, [(33, 2)]), (192, [(200, 2), (0, 1), (0, 0), (194, 1)])],
])
def test_sequences_that_may_not_share_between_members(groups, hd, nq, nkv, bits):
    check(groups, nq, nkv, hd, bits, seed=21)


def test_many_sequences_between_members():
    check([(64, [(66, 1) if i % 11 == 0 else (40, 1) for i in range(700)]), (64, [(200, 1)] + [(60, 2)] * 300 + [(70, 2)])], 2, 1, 64, 16, seed=22)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("hd, nq, nkv", HEADS)
@pytest.mark.parametrize("times", [1, 30])
@pytest.mark.parametrize("cu, lens, queries", DECREASING)
def test_decreasing_tokens_inside_a_group_write_nothing_else(cu, lens, queries, times, hd, nq, nkv, bits):
    """Results are not defined then, but rows of no sequence and what lies around the workspace stay as they are."""
    more = 2 * (times - 1)
    cu = [2 * i for i in range(times - 1)] + [more + x for x in cu]
    lens = [140] * (times - 1) + lens
    (cache, c, tables, _, _, q), starts, shared, _ = make_groups([(128, [(200, 1)] * len(lens))], nq, nkv, hd, bits, seed=23)
    T = max(cu) + 2
    q = dev((np.random.default_rng(24).standard_normal((T, nq, hd)) / np.sqrt(hd)).astype(np.float16))
    out = torch.full((T + 2, nq, hd), 9.0, dtype=torch.float16, device="cuda")
    n = B.shared_attention_workspace_bytes(nq, cache, len(lens), 1, T, 20)
    work = torch.full((n + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    work[:8192] = 0
    B.shared_attention(q, cache, dev(tables), dev(np.int32(lens)), dev(np.int32(cu)), dev(starts), dev(shared), out[:T], work[:n], max_q=20, share_all=True)
    assert (out[max(cu):] == 9.0).all() and (work[n:] == 0xA5).all() and not work[:8192].any()
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("members", [2, 40])
def test_context_lengths_that_do_not_fit(members, bits):
    """Contexts beyond the table's width end there, negative ones are empty; the groups' tokens are in order."""
    b, starts, shared, max_q = make_groups([(128, [(140, 1)] * members), (70, [(80, 2), (75, 1)])], 4, 2, 64, bits, seed=25, extra_rows=2)
    cache, c, tables, lens, cu, q = b
    given, seen = lens.copy(), lens.copy()
    for s, n in ((0, 2 ** 31 - 1), (1, -5), (members, -2 ** 31), (members + 1, 2 ** 31 - 1)):
        given[s] = n
        seen[s] = tables.shape[1] * 16 if n > 0 else 0
    for s in (0, members + 1):                         # (blocks for all of it)
        tables[s, (lens[s] + 15) // 16:] = tables[s, 0]
    got = run_shared((cache, c, tables, given, cu, q), starts, shared, max_q)
    check_attention(got, cache, c, tables, seen, cu, q)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("hd, nq, nkv", HEADS)
@pytest.mark.parametrize("before, after", [
    ([(60, 1)] * 30, [(90, 1)] * 30),                        # in no group
    ([(333, 333)], [(150, 40), (77, 1)]),                    # prompts, more rows than the few-row part holds
    ([(50, 3), (70, 5), (20, 1)], [(100, 8)] * 3),           # drafts
    ([(400, 70)], [(60, 4)] * 20 + [(0, 1)]),
])
def test_groups_beside_others(before, after, hd, nq, nkv, bits):
    check([(130, [(135 + i, 1) for i in range(3)]), (100, [(104, 4), (101, 1)]), (70, [(71, 1)] * 30)], nq, nkv, hd, bits, seed=26, before=before, after=after)


def test_workspace_does_not_grow_with_prompts():
    """Only sequences of fewer than 256 rows have results to be joined: a prompt's tokens take a note of 32 bytes each, and no rows."""
    cache = make_groups([(64, [(70, 1), (71, 1)])], 32, 8, 128, 16)[0][0]
    size = lambda seqs, tokens, max_q: B.shared_attention_workspace_bytes(32, cache, seqs, 1, tokens, max_q)      # noqa: E731
    assert size(33, 65568, 65536) - size(33, 16416, 16384) == 32 * (65568 - 16416)
    assert size(33, 16416, 16384) - size(33, 33, 1) <= 32 * 16416 + 2 * 33 * 63 * 32 * 132 * 4
    for seqs, tokens, max_q in ((33, 16416, 16384), (1000, 1000, 1), (40, 400, 17), (7, 3000, 2999)):
        for fewer in ((seqs - 1, tokens, max_q), (seqs, tokens - 1, max_q), (seqs, tokens, max(1, max_q // 2)), (1, tokens, max_q), (seqs, 1, max_q)):
            assert size(*fewer) <= size(seqs, tokens, max_q)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("window, sinks", [(150, 0), (190, 5), (191, 0), (260, 17), (500, 16)])
@pytest.mark.parametrize("hd, nq, nkv", [(64, 4, 2), (128, 8, 2)])
@pytest.mark.parametrize("members", [
    [(130 + i, 1) for i in range(40)] + [(400, 1)],          # more rows than the few-row part holds
    [(170, 40), (260, 70), (189, 61), (190, 1)],             # prompt items behind the shared keys, which end before the window is left, with it and behind it
    [(190 + i, 1 + 9 * (i % 5)) for i in range(20)],
])
def test_windows_behind_groups_of_many_rows(members, hd, nq, nkv, window, sinks, bits):
    check([(128, members)], nq, nkv, hd, bits, window=window, sinks=sinks, seed=27)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("groups", [
    [(128, [(140 + i, 1) for i in range(40)])],              # runs of shared keys
    [(128, [(140, 1), (3000, 40), (2900, 3)])],              # a prompt's parts joined
    [(128, [(140, 1), (500, 300), (135, 2)])],               # and one without rows among its members
])
def test_strided_rows(groups, bits):
    b, starts, shared, max_q = make_groups(groups, 4, 2, 64, bits, seed=28)
    cache, c, tables, lens, cu, q = b
    T = q.shape[0]
    wide_q, wide_o = torch.zeros(T, 9, 64, dtype=torch.float16, device="cuda"), torch.full((T, 7, 64), 3.0, dtype=torch.float16, device="cuda")
    wide_q[:, 2:6] = dev(q)
    work = torch.zeros(B.shared_attention_workspace_bytes(4, cache, len(lens), 1, T, max_q), dtype=torch.uint8, device="cuda")
    B.shared_attention(wide_q[:, 2:6], cache, dev(tables), dev(lens), dev(cu), dev(starts), dev(shared), wide_o[:, 1:5], work, max_q=max_q, share_all=True)
    o = wide_o.cpu().numpy()
    check_attention(o[:, 1:5].astype(np.float64), *b)
    assert (o[:, :1] == 3).all() and (o[:, 5:] == 3).all()


def test_repeated_calls_are_the_same_to_the_last_bit():
    """Whichever workgroup comes first, sums are in the order of the runs: groups in runs and in parts, drafts, prompts, all in one batch, twenty times."""
    for bits in (16, 4):
        b, starts, shared, max_q = make_groups([(400, [(410 + i, 1) for i in range(50)]), (300, [(320, 20), (900, 300), (330, 12)]), (64, [(70, 5), (66, 1)])], 8, 2, 128, bits, seed=29,
                                               before=[(700, 1)], after=[(500, 120), (30, 1)])
        got = run_shared(b, starts, shared, max_q)
        check_attention(got, *b)
        for _ in range(20):
            assert np.array_equal(got, run_shared(b, starts, shared, max_q))
