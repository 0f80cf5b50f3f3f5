"""Argument checks of the rotary and 4-bit cache entry points (no GPU): every
call below returns before any HIP runtime call is made."""
import ctypes
import math
import os

import pytest
import torch

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


def test_record_bytes(K):
    L = K.lib()
    assert L.gvr_kv4_record_bytes(8, 128) == 1088 and L.gvr_kv4_record_bytes(1, 64) == 68
    assert L.gvr_kv4_record_bytes(3, 256) == 816
    for h, d in ((0, 128), (-1, 128), (1025, 128), (8, 96), (8, 0), (8, 512)):
        assert L.gvr_kv4_record_bytes(h, d) == -1
        with pytest.raises(ValueError):
            K.gvr_kv4_record_bytes(h, d)


def test_rope_table_checks(K):
    L = K.lib()
    import paper_2604_22312_amd as g
    assert L.gvr_rope_table(0, None, 1.0, None, None) == 0
    assert L.gvr_rope_table(-1, None, 1.0, vp(64), None) == -1
    assert L.gvr_rope_table(5, None, 1.0, None, None) == -1
    assert L.gvr_rope_table(5, None, math.inf, vp(64), None) == -1
    assert L.gvr_rope_table(5, None, math.nan, vp(64), None) == -1
    assert L.gvr_rope_table(5, None, 1.0, vp(68), None) == -1
    assert L.gvr_rope_table(1 << 31, None, 1.0, vp(64), None) == -5
    assert L.gvr_rope_table(5, ctypes.byref(g.gvr_rope_params(d_rope=63)), 1.0, vp(64), None) == -1


def test_rope_rotate_checks(K):
    L = K.lib()

    def call(T=4, H=2, D=64, dtype=0, x=256, o=512, pos=64, cs=(64, 100, 64, 0)):
        xs, os_ = K._Heads(x, H * D, D), K._Heads(o, H * D, D)
        c = K._RopeCs(*cs) if cs else None
        return L.gvr_rope_rotate(ctypes.byref(xs), ctypes.byref(os_), dtype, T, H, D, vp(pos) if pos else None,
                                 ctypes.byref(c) if c else None, None)
    assert call(T=0) == 0 and call(H=0) == 0
    assert call(T=0, x=0, o=0, pos=0) == 0
    for kw in (dict(T=-1), dict(H=-1), dict(D=0), dict(D=2048), dict(dtype=3), dict(dtype=-1), dict(x=0), dict(o=0),
               dict(pos=0), dict(cs=None), dict(x=257), dict(o=514, dtype=2),
               dict(cs=(64, 100, 66, 0)), dict(cs=(64, 100, 0, 0)), dict(cs=(64, 100, 7, 0)), dict(cs=(64, -1, 64, 0)),
               dict(cs=(0, 100, 64, 0)), dict(cs=(68, 100, 64, 0)), dict(cs=(64, 100, 64, 4))):
        assert call(**kw) == -1, kw
    assert call(T=1 << 31) == -5 and call(H=1 << 21) == -5


def _cache(K, data=4096, pages=4, page=16, heads=2, D=64, reserved=0):
    return K._Cache(data, pages, page, heads, D, reserved)


BAD_CACHES = (dict(pages=-1), dict(page=0), dict(page=48), dict(page=131072), dict(heads=0), dict(D=80),
              dict(reserved=1), dict(data=0), dict(data=4097))


def test_append_and_read_checks(K):
    L = K.lib()

    def append(T=3, dtype=0, k=256, v=512, slots=64, pos=None, cs=None, **c):
        cache, ks, vs = _cache(K, **c), K._Heads(k, 128, 64), K._Heads(v, 128, 64)
        t = K._RopeCs(*cs) if cs else None
        return L.gvr_kv4_append(ctypes.byref(cache), ctypes.byref(ks), ctypes.byref(vs), dtype, T,
                                vp(slots) if slots else None, vp(pos) if pos else None,
                                ctypes.byref(t) if t else None, None)

    def read(T=3, dtype=0, k=256, v=512, slots=64, **c):
        cache, ks, vs = _cache(K, **c), K._Heads(k, 128, 64), K._Heads(v, 128, 64)
        return L.gvr_kv4_read(ctypes.byref(cache), ctypes.byref(ks), ctypes.byref(vs), dtype, T,
                              vp(slots) if slots else None, None)
    for f in (append, read):
        assert f(T=0) == 0 and f(T=0, data=0, slots=0) == 0
        for kw in BAD_CACHES + (dict(T=-1), dict(dtype=3), dict(slots=0), dict(k=257), dict(v=513)):
            assert f(**kw) == -1, kw
        assert f(T=1 << 31) == -5 and f(pages=1 << 31) == -5 and f(pages=1 << 28) == -5
    assert append(k=0) == -1 and append(v=0) == -1
    assert read(k=0, v=0) == 0
    assert L.gvr_kv4_append(ctypes.byref(_cache(K)), None, None, 0, 0, None, None, None, None) == -1
    assert append(cs=(64, 10, 64, 0)) == -1                       # no positions
    assert append(cs=(64, 10, 128, 0), pos=64) == -1              # rotates more than a head
    assert append(cs=(64, 10, 64, K.ROPE_TRANSPOSED), pos=64) == -1
    assert L.gvr_kv4_append(None, ctypes.byref(K._Heads(256, 128, 64)), ctypes.byref(K._Heads(256, 128, 64)), 0, 0, None,
                            None, None, None) == -1


def test_attention_checks(K):
    L = K.lib()
    base = dict(q=256, q_token_stride=256, q_head_stride=64, out=512, lse=None, block_table=64, ctx_len=64, q_start=None,
                selection=None, T=4, table_width=8, sequences=2, max_q=0, q_heads=4, K=0, dtype=0, causal=1, scale=0.1,
                reserved=0)

    def call(ws=(0, 0), cache=None, **kw):
        a = dict(base)
        a.update(kw)
        arg = K._AttentionArgs(**a)
        c = _cache(K, **(cache or {}))
        return L.gvr_kv4_attention(ctypes.byref(c), ctypes.byref(arg), vp(ws[0]) if ws[0] else None, ws[1], None)
    assert call(T=0, q=None, out=None, ctx_len=None, block_table=None) == 0
    assert call(T=0, sequences=0) == 0
    for kw in (dict(T=-1), dict(sequences=-1), dict(table_width=-1), dict(q_heads=0), dict(q_heads=3), dict(q_heads=258),
               dict(dtype=2), dict(dtype=-1), dict(causal=2), dict(scale=math.inf), dict(scale=math.nan),
               dict(reserved=1), dict(q_token_stride=12), dict(q_head_stride=4), dict(selection=64, K=0),
               dict(T=5), dict(q_start=64, max_q=-1), dict(q=None), dict(out=None), dict(ctx_len=None),
               dict(block_table=None), dict(q=264), dict(out=520), dict(ws=(0, 64)), dict(ws=(8, 64))):
        assert call(**kw) == -1, kw
    for c in BAD_CACHES:
        assert call(cache=c) == -1, c
    assert call(T=1 << 31, sequences=1 << 30) == -5 and call(table_width=1 << 28) == -5
    n = ctypes.c_size_t(7)
    arg = K._AttentionArgs(**base)
    assert L.gvr_kv4_attention_workspace(ctypes.byref(_cache(K)), ctypes.byref(arg), None) == -1
    assert L.gvr_kv4_attention_workspace(None, ctypes.byref(arg), ctypes.byref(n)) == -1
    assert L.gvr_kv4_attention_workspace(ctypes.byref(_cache(K)), None, ctypes.byref(n)) == -1
    arg.T = 0
    assert L.gvr_kv4_attention_workspace(ctypes.byref(_cache(K, data=0)), ctypes.byref(arg), ctypes.byref(n)) == 0
    assert n.value == 0


def test_binding_refuses_cpu_tensors(K):
    x = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        K.gvr_rope_rotate(x, torch.zeros(2, dtype=torch.int32), torch.zeros(4, 32, 2))
    with pytest.raises(ValueError):
        K.gvr_kv4_append(x, x, torch.zeros(2, dtype=torch.int64), torch.zeros(1, 16, 136, dtype=torch.uint8))
    with pytest.raises(ValueError):
        K.gvr_kv4_read(torch.zeros(1, 16, 136, dtype=torch.uint8), torch.zeros(2, dtype=torch.int64), 2, 64)
    with pytest.raises(ValueError):
        K.gvr_kv4_attention(x, torch.zeros(1, 16, 136, dtype=torch.uint8), torch.zeros(2, 1, dtype=torch.int32),
                            torch.zeros(2, dtype=torch.int32), 2)
    with pytest.raises(ValueError):
        K.gvr_rope_table(10, device="cpu")
