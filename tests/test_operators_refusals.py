"""What the operators on device memory refuse, before any device is asked for (no GPU needed)."""
import ctypes as C

import pytest

import paper_2604_07609_amd as B
from paper_2604_07609_amd import binding as M

P = 1 << 20        # an aligned address that nothing reads


def cache(**k):
    return M.CacheDesc(**{**dict(data=P, n_blocks=4, n_kv_heads=2, head_dim=64, bits=16), **k})


def store(**k):
    c = k.pop("cache", cache())
    return M.QkNormRopeArgs(**{**dict(cache=c, n_q_heads=4, n_tokens=3, in_type=1, rope_rows=8, q=P, k=P, v=P, q_stride=256, k_stride=128, v_stride=128, q_gain=P, k_gain=P,
                                      positions=P, slots=P, rope_table=P, q_out=P, q_out_stride=256, eps=1e-6, q_scale=1.0), **k})


def attend(**k):
    c = k.pop("cache", cache())
    return M.PagedAttentionArgs(**{**dict(cache=c, n_q_heads=4, n_seqs=2, n_tokens=2, max_q=1, max_blocks=4, window=8, sinks=2, scale=1.0, q=P, out=P, q_stride=256, out_stride=256,
                                          cu_seqlens=P, seq_lens=P, block_tables=P, workspace=P, workspace_bytes=1 << 30), **k})


BAD_CACHES = [dict(data=None), dict(data=P + 64), dict(bits=8), dict(bits=0), dict(head_dim=96), dict(n_blocks=0), dict(n_kv_heads=0), dict(n_kv_heads=3), dict(n_kv_heads=2000)]


@pytest.mark.parametrize("bad", BAD_CACHES + [dict(n_blocks=(1 << 27) + 1)])
def test_caches(bad):
    lib = B.load_library()
    want = B.ERR_TOO_LARGE if bad.get("n_blocks", 0) > 1 << 27 else B.ERR_INVAL
    assert lib.blink_qk_norm_rope(0, C.byref(store(cache=cache(**bad))), None) == want
    assert lib.blink_last_error()
    assert lib.blink_paged_attention(0, C.byref(attend(cache=cache(**bad))), None) == want
    if "n_kv_heads" not in bad or bad["n_kv_heads"] in (0, 2000):
        assert lib.blink_kv_cache_read(0, C.byref(cache(**bad)), P, 3, P, P, None) == want


@pytest.mark.parametrize("bad", [dict(n_q_heads=0), dict(n_q_heads=5), dict(n_q_heads=130), dict(in_type=3), dict(rope_rows=0), dict(q=None), dict(k=None), dict(v=None), dict(q=P + 8),
                                 dict(k=P + 2), dict(q_stride=255), dict(q_stride=248), dict(k_stride=120), dict(v_stride=0), dict(v_stride=132), dict(q_out=None), dict(q_out=P + 4),
                                 dict(q_out_stride=8), dict(positions=None), dict(slots=None), dict(slots=P + 2), dict(rope_table=None), dict(rope_table=P + 8), dict(q_gain=P + 4),
                                 dict(k_gain=P + 8), dict(eps=-1.0), dict(eps=float("nan"))])
def test_qk_norm_rope(bad):
    lib = B.load_library()
    assert lib.blink_qk_norm_rope(0, C.byref(store(**bad)), None) == B.ERR_INVAL
    assert lib.blink_last_error()


@pytest.mark.parametrize("bad", [dict(n_q_heads=0), dict(n_q_heads=3), dict(n_q_heads=130), dict(max_q=0), dict(max_q=1 << 24), dict(max_blocks=0), dict(max_blocks=1 << 27), dict(scale=0.0),
                                 dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(window=0), dict(window=1 << 31), dict(sinks=1 << 31), dict(q=None), dict(out=None),
                                 dict(q=P + 8), dict(out=P + 8), dict(q_stride=128), dict(out_stride=260), dict(cu_seqlens=None), dict(seq_lens=None), dict(block_tables=None),
                                 dict(cu_seqlens=P + 1)])
def test_paged_attention(bad):
    lib = B.load_library()
    assert lib.blink_paged_attention(0, C.byref(attend(**bad)), None) == B.ERR_INVAL
    assert lib.blink_last_error()


def test_too_large():
    lib = B.load_library()
    assert lib.blink_paged_attention(0, C.byref(attend(n_seqs=1025)), None) == B.ERR_TOO_LARGE
    assert lib.blink_paged_attention(0, C.byref(attend(n_seqs=1024, max_blocks=1 << 21)), None) == B.ERR_TOO_LARGE
    assert lib.blink_paged_attention(0, C.byref(attend(n_tokens=1 << 30)), None) == B.ERR_TOO_LARGE
    assert lib.blink_qk_norm_rope(0, C.byref(store(n_tokens=1 << 29)), None) == B.ERR_TOO_LARGE


def test_nothing_to_do_is_no_error():
    lib = B.load_library()
    assert lib.blink_qk_norm_rope(0, C.byref(store(n_tokens=0)), None) == 0
    assert lib.blink_paged_attention(0, C.byref(attend(n_seqs=0)), None) == 0
    assert lib.blink_paged_attention(0, C.byref(attend(n_tokens=0)), None) == 0
    assert lib.blink_kv_cache_read(0, C.byref(cache()), None, 0, None, None, None) == 0


def test_null_arguments():
    lib, n = B.load_library(), C.c_uint64()
    assert lib.blink_qk_norm_rope(0, None, None) == B.ERR_INVAL and lib.blink_paged_attention(0, None, None) == B.ERR_INVAL
    assert lib.blink_kv_cache_read(0, None, P, 3, P, P, None) == B.ERR_INVAL
    for bad in ((None, P, P), (P, None, P), (P, P, None), (P + 2, P, P), (P, P + 8, P)):
        assert lib.blink_kv_cache_read(0, C.byref(cache()), bad[0], 3, bad[1], bad[2], None) == B.ERR_INVAL
    assert lib.blink_kv_cache_bytes(4, 2, 64, 16, None) == B.ERR_INVAL and lib.blink_attention_workspace_bytes(0, None, 4, 2, 1, C.byref(n)) == B.ERR_INVAL
    assert lib.blink_attention_workspace_bytes(0, C.byref(cache()), 4, 2000, 1, C.byref(n)) == B.ERR_TOO_LARGE


@pytest.mark.parametrize("hd", [64, 128])
def test_cache_bytes(hd):
    assert B.kv_cache_bytes(5, 3, hd) == 2 * 5 * 3 * 16 * hd * 2
    assert B.kv_cache_bytes(5, 3, hd, 4) == 5 * 3 * (16 * hd + 16 * 2 * hd // 32)
    with pytest.raises(B.BlinkError):
        B.kv_cache_bytes(0, 3, hd)


def test_struct_sizes_match_header(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "blink.h"\nint main(void) { printf("%zu %zu %zu %zu %zu\\n", sizeof(blink_kv_cache), '
                   'sizeof(blink_qk_norm_rope_args), offsetof(blink_qk_norm_rope_args, eps), sizeof(blink_paged_attention_args), offsetof(blink_paged_attention_args, workspace)); return 0; }\n')
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(root, "include"), "-o", str(exe), str(src)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [C.sizeof(M.CacheDesc), C.sizeof(M.QkNormRopeArgs), M.QkNormRopeArgs.eps.offset, C.sizeof(M.PagedAttentionArgs), M.PagedAttentionArgs.workspace.offset]


@pytest.mark.parametrize("kind, form", [(M.CacheDesc, "_CACHE"), (M.QkNormRopeArgs, "_QK_NORM_ROPE"), (M.PagedAttentionArgs, "_PAGED_ATTENTION")])
def test_packed_arguments_are_the_structures(kind, form):
    """The binding packs its arguments with `struct`: every field where the structure has it."""
    packer = getattr(M, form)
    n = len(packer.unpack(bytes(packer.size)))
    got = kind.from_buffer_copy(packer.pack(*range(1, n + 1)).ljust(C.sizeof(kind), b"\0"))
    flat = []
    for name, _ in kind._fields_:
        x = getattr(got, name)
        flat += [getattr(x, f) for f, _ in x._fields_] if isinstance(x, C.Structure) else [x]
    assert [int(x) for x in flat] == list(range(1, n + 1)) and packer.size <= C.sizeof(kind)


def test_tensors_of_the_wrong_kind():
    """The binding's own checks, on host tensors: they are on no device of the library's."""
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError, match="data is on cpu"):
        B.KVCache(torch.zeros(B.kv_cache_bytes(2, 1, 64), dtype=torch.uint8), 2, 1, 64)
