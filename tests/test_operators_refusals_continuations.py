"""What the operators for continuations of one prompt refuse, before any device is asked for (no GPU needed)."""
import ctypes as C

import pytest
import torch

import paper_2604_07609_amd as B
from paper_2604_07609_amd import binding as M
from tests.test_operators_refusals import P, attend, cache


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


def groups(**k):
    own = {n: k.pop(n) for n in ("n_groups", "share_all", "group_starts", "shared_lens") if n in k}
    return M.SharedAttentionArgs(**{**dict(attention=attend(**k), n_groups=2, share_all=0, group_starts=P, shared_lens=P), **own})


@pytest.mark.parametrize("bad", [dict(share_all=2), dict(group_starts=None), dict(shared_lens=None), dict(group_starts=P + 2), dict(shared_lens=P + 1), dict(n_q_heads=3), dict(max_q=0), dict(max_blocks=0),
                                 dict(scale=0.0), dict(window=0), dict(q=None), dict(out=P + 8), dict(q_stride=128), dict(seq_lens=None), dict(block_tables=P + 1), dict(cache=cache(bits=8)),
                                 dict(cache=cache(head_dim=96)), dict(cache=cache(data=None)), dict(n_groups=0, q=None), dict(n_groups=0, scale=-1.0)])
def test_shared_attention(bad):
    lib = B.load_library()
    assert lib.blink_shared_attention(0, C.byref(groups(**bad)), None) == B.ERR_INVAL
    assert lib.blink_last_error()


def test_shared_attention_too_large_none_and_nothing():
    lib, n = B.load_library(), C.c_uint64()
    call = lambda **k: lib.blink_shared_attention(0, C.byref(groups(**k)), None)      # noqa: E731
    assert lib.blink_shared_attention(0, None, None) == B.ERR_INVAL
    assert call(n_seqs=0) == 0 and call(n_tokens=0, group_starts=None) == 0
    assert call(n_seqs=1000, n_groups=25) == B.ERR_TOO_LARGE and call(n_seqs=2, n_groups=(1 << 32) - 1) == B.ERR_TOO_LARGE and call(n_seqs=1025, n_groups=0) == B.ERR_TOO_LARGE
    assert call(n_tokens=1 << 29) == B.ERR_TOO_LARGE
    assert call(n_seqs=512, n_groups=512, max_blocks=1 << 20) == B.ERR_TOO_LARGE                       # 2 kv heads: 2^31 blocks with the groups' own, half of that without
    # the results are joined by a wave per token and four heads of 64, or two of 128: 2^26 waves are 2^32 threads
    assert call(n_tokens=1 << 26, n_q_heads=4) == B.ERR_TOO_LARGE and b"tokens" in lib.blink_last_error()
    assert call(n_tokens=1 << 25, n_q_heads=4, cache=cache(head_dim=128), q_stride=512, out_stride=512) == B.ERR_TOO_LARGE
    size = lambda c, *k: lib.blink_shared_attention_workspace_bytes(0, c and C.byref(c), *k)           # noqa: E731
    assert size(None, 4, 2, 1, 8, 1, C.byref(n)) == B.ERR_INVAL and size(cache(), 4, 2, 1, 8, 1, None) == B.ERR_INVAL and size(cache(), 3, 2, 1, 8, 1, C.byref(n)) == B.ERR_INVAL


def test_structures_of_the_continuations_match_the_header(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "blink.h"\nint main(void) { printf("%zu %zu %zu %zu %zu\\n", sizeof(blink_shared_attention_args), '
                   'offsetof(blink_shared_attention_args, n_groups), offsetof(blink_shared_attention_args, shared_lens), sizeof(blink_token_logprobs_args), '
                   'offsetof(blink_token_logprobs_args, workspace_bytes)); return 0; }\n')
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(root, "include"), "-o", str(exe), str(src)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [C.sizeof(M.SharedAttentionArgs), M.SharedAttentionArgs.n_groups.offset, M.SharedAttentionArgs.shared_lens.offset, C.sizeof(M.TokenLogprobsArgs),
                   M.TokenLogprobsArgs.workspace_bytes.offset]


def test_packed_arguments_of_the_continuations_are_the_structures():
    n = len(M._TOKEN_LOGPROBS.unpack(bytes(M._TOKEN_LOGPROBS.size)))
    got = M.TokenLogprobsArgs.from_buffer_copy(M._TOKEN_LOGPROBS.pack(*range(1, n + 1)))
    assert [int(getattr(got, f)) for f, _ in got._fields_] == list(range(1, n + 1))
    m = len(M._PAGED_ATTENTION.unpack(bytes(M._PAGED_ATTENTION.size)))
    got = M.SharedAttentionArgs.from_buffer_copy(M._PAGED_ATTENTION.pack(*range(1, m + 1)) + M._GROUPS.pack(*range(m + 1, m + 5)))
    assert [int(getattr(got, f)) for f, _ in got._fields_[1:]] == list(range(m + 1, m + 5)) and got.attention.workspace_bytes == m
