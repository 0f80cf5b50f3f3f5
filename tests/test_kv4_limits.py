"""Limits of the rotary and 4-bit cache entry points (no GPU): every call below
returns before anything would be launched."""
import ctypes
import os

import pytest

vp = ctypes.c_void_p


@pytest.fixture(scope="module")
def K():
    import paper_2604_22312_amd as g
    if not os.path.exists(g.library_path()):
        from paper_2604_22312_amd import build
        build.build()
    from paper_2604_22312_amd import kv4
    kv4.lib()
    return kv4


def attention(lib, page=16, heads=2, D=64, pages=4, **kw):
    a = dict(q=256, q_token_stride=256, q_head_stride=64, out=512, lse=None, block_table=64, ctx_len=64, q_start=None,
             selection=None, T=4, table_width=8, sequences=2, max_q=0, q_heads=4, K=0, dtype=0, causal=1, scale=0.1,
             reserved=0)
    a.update(kw)
    arg, c = lib._AttentionArgs(**a), lib._Cache(4096, pages, page, heads, D, 0)
    return lib.lib().gvr_kv4_attention(ctypes.byref(c), ctypes.byref(arg), None, 0, None)


def test_no_query_tokens_to_serve(K):
    """max_q = 0: no sequence has a row that is served, so nothing is launched."""
    assert attention(K, q_start=64, max_q=0) == 0
    assert attention(K, q_start=64, max_q=0, selection=64, K=5) == 0
    n = ctypes.c_size_t(7)
    arg = K._AttentionArgs(q_start=64, T=4, table_width=8, sequences=2, q_heads=4, scale=0.1)
    assert K.lib().gvr_kv4_attention_workspace(ctypes.byref(K._Cache(4096, 4, 16, 2, 64, 0)), ctypes.byref(arg),
                                               ctypes.byref(n)) == 0 and n.value == 0


def test_more_threads_than_a_launch_holds(K):
    """2^23 workgroups of 512 threads (2^24 of 256 at D = 256): refused before the launch."""
    far = dict(q_start=64, pages=1000)
    assert attention(K, selection=64, K=2048, sequences=1024, T=16384, max_q=16384, **far) == -5
    assert attention(K, selection=64, K=5, sequences=1, T=1 << 23, max_q=1 << 23, heads=8, q_heads=8, **far) == -5
    assert attention(K, sequences=1 << 14, T=1 << 19, max_q=1 << 19, **far) == -5
    assert attention(K, sequences=1 << 13, T=1 << 19, max_q=1 << 19, D=256, **far) == -5


def test_heads_of_a_rotation(K):
    """2^20 heads at most, as gvr_rotary.h says."""
    xs, cs = K._Heads(256, 64, 64), K._RopeCs(64, 100, 64, 0)
    for H, want in ((1 << 20, 0), ((1 << 20) + 1, -5)):
        assert K.lib().gvr_rope_rotate(ctypes.byref(xs), ctypes.byref(xs), 0, 0, H, 64, vp(64), ctypes.byref(cs), None) == want
    header = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "gvr_rotary.h")
    assert "H above 2^20" in open(header).read()
