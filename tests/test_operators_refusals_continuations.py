"""What the operators for continuations of one prompt refuse, before any device is asked for (no GPU needed)."""
import ctypes as C

import pytest
import torch

import paper_2604_07609_amd as B
from paper_2604_07609_amd import binding as M
from tests.test_operators_refusals import P, cache


def logprobs(**k):
    return M.TokenLogprobsArgs(**{**dict(type=0, n_rows=3, vocab=100, n_given=2, k=4, logits=P, stride=100, tokens=P, inverse_temperature=P, logprobs=P, ranks=P, entropy=P, top_ids=P,
                                         top_logprobs=P, workspace=P, workspace_bytes=1 << 30), **k})


@pytest.mark.parametrize("bad", [dict(type=3), dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(n_given=65), dict(k=65), dict(k=101, vocab=100), dict(logits=None), dict(logits=P + 2),
                                 dict(logits=P + 1, type=1), dict(stride=99), dict(tokens=None), dict(logprobs=None), dict(top_ids=None), dict(top_logprobs=None), dict(tokens=P + 2),
                                 dict(ranks=P + 1), dict(entropy=P + 2), dict(top_ids=P + 3), dict(top_logprobs=P + 2), dict(inverse_temperature=P + 1)])
def test_token_logprobs(bad):
    lib = B.load_library()
    assert lib.blink_token_logprobs(0, C.byref(logprobs(**bad)), None) == B.ERR_INVAL
    assert lib.blink_last_error()


def test_token_logprobs_too_large_none_and_nothing():
    lib, n = B.load_library(), C.c_uint64()
    assert lib.blink_token_logprobs(0, None, None) == B.ERR_INVAL
    assert lib.blink_token_logprobs(0, C.byref(logprobs(n_rows=1 << 25)), None) == B.ERR_TOO_LARGE
    assert lib.blink_token_logprobs(0, C.byref(logprobs(n_rows=0, logits=None)), None) == 0
    assert lib.blink_token_logprobs_workspace_bytes(0, 3, 100, 2, 4, None) == B.ERR_INVAL
    assert lib.blink_token_logprobs_workspace_bytes(0, 3, 100, 65, 4, C.byref(n)) == B.ERR_INVAL
    assert lib.blink_token_logprobs_workspace_bytes(0, 1 << 25, 100, 2, 4, C.byref(n)) == B.ERR_TOO_LARGE


def copy(lib, caches, n=None, source=P, to=P, copies=3):
    a = (M.CacheDesc * max(1, len(caches)))(*caches)
    return lib.blink_kv_cache_copy(0, C.byref(a), len(caches) if n is None else n, source, to, copies, None)


@pytest.mark.parametrize("bad", [dict(data=None), dict(data=P + 64), dict(bits=8), dict(head_dim=96), dict(n_blocks=0), dict(n_kv_heads=0)])
def test_kv_cache_copy_caches(bad):
    lib = B.load_library()
    assert copy(lib, [cache(**bad)]) == B.ERR_INVAL and lib.blink_last_error()
    assert copy(lib, [cache(), cache(**bad)]) == B.ERR_INVAL


@pytest.mark.parametrize("unlike", [dict(n_blocks=5), dict(n_kv_heads=4), dict(head_dim=128), dict(bits=4)])
def test_kv_cache_copy_caches_unlike_the_first(unlike):
    lib = B.load_library()
    assert copy(lib, [cache(), cache(**unlike)]) == B.ERR_INVAL and b"first" in lib.blink_last_error()


def test_kv_cache_copy():
    lib = B.load_library()
    for source, to in ((None, P), (P, None), (P + 2, P), (P, P + 1)):
        assert copy(lib, [cache()], source=source, to=to) == B.ERR_INVAL
    assert lib.blink_kv_cache_copy(0, None, 1, P, P, 1, None) == B.ERR_INVAL
    assert copy(lib, [cache()], copies=0, source=None, to=None) == 0
    assert lib.blink_kv_cache_copy(0, None, 0, None, None, 3, None) == 0
    assert copy(lib, [cache()], copies=1 << 24) == B.ERR_TOO_LARGE


def test_the_binding_refuses_tensors_that_do_not_fit():
    x, w = torch.zeros(3, 50), torch.zeros(100, dtype=torch.uint8)
    with pytest.raises(ValueError, match="on a GPU"):
        B.token_logprobs(x, w)
    with pytest.raises(ValueError, match="two dimensions"):
        B.token_logprobs(x[0], w)
    with pytest.raises(ValueError, match="float32, float16 or bfloat16"):
        B.token_logprobs(x.double(), w)
