"""A sequence's rows do not depend on the batch that it is in by more than rounding: alone, among few and many others, with prompts beside it."""
import numpy as np
import pytest
import torch

import paper_2604_07609_amd as B
from tests.test_gpu_operators import check_attention, make_batch, no_error_of_earlier_tests  # noqa: F401
from tests.test_gpu_operators_workspace import attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("hd, nq, nkv", [(64, 8, 8), (128, 4, 1)])
@pytest.mark.parametrize("n, run, window, sinks", [(1300, 1, 0, 0), (1300, 3, 300, 5), (40, 1, 0, 0)])
def test_one_sequence_in_batches_of_many_kinds(n, run, window, sinks, hd, nq, nkv, bits):
    """How runs of tiles are cut, whether pairs are dealt out whole, and who adds results up depend on the rest of the batch."""
    cache, c, tables, lens, cu, q = make_batch([n, 700, 33], [run, 40, 1], nq, nkv, hd, bits, seed=91)
    mine = q[:run]
    one = (cache, c, tables[:1], lens[:1], np.int32([0, run]), mine)
    mask = dict(window=window, sinks=sinks)
    work = torch.zeros(B.attention_workspace_bytes(nq, cache, 1024, 40), dtype=torch.uint8, device="cuda")
    check_attention(attend(one, run, mask, work).double().cpu().numpy(), *one, **mask)
    rng = np.random.default_rng(92)
    for others, at, prompt in ((1, 0, False), (3, 2, False), (40, 17, False), (63, 63, False), (64, 5, False), (200, 100, False), (700, 650, False), (2, 1, True), (90, 45, True)):
        t, m, r, x = [], [], [], []
        for s in range(others + 1):
            if s == at:
                t.append(tables[0]); m.append(n); r.append(run); x.append(mine)
                continue
            k = 40 if prompt and s % 3 == 0 else 1
            t.append(tables[1]); m.append(int(rng.integers(k, 701))); r.append(k); x.append(rng.standard_normal((k, nq, hd)).astype(np.float16))
        starts = np.concatenate(([0], np.cumsum(r))).astype(np.int32)
        got = attend((cache, c, np.stack(t), np.int32(m), starts, np.concatenate(x)), max(r), mask, work)[starts[at]:starts[at] + run]
        check_attention(got.double().cpu().numpy(), *one, **mask)    # (against the oracle, in the tolerance of the sequence alone)
