"""Argument checks of the 8-bit matrices' and the page step's entry points (no GPU): every call below returns before any
HIP runtime call is made."""
import ctypes
import os

import pytest
import torch

vp = ctypes.c_void_p


@pytest.fixture(scope="module")
def F():
    import paper_2604_22312_amd as g
    if not os.path.exists(g.library_path()):
        from paper_2604_22312_amd import build
        build.build()
    from paper_2604_22312_amd import fp8
    fp8.lib()
    return fp8


@pytest.fixture(scope="module")
def P(F):
    from paper_2604_22312_amd import pages
    pages.lib()
    return pages


def test_quantize_checks(F):
    L = F.lib()

    def call(dtype=0, T=4, H=2, D=128, x=256, pos=None, cs=None, out=(512, 256, 128, 1024, 2, 1), slots=None, rows=9, flags=0):
        xs, os_ = F._Heads(x, H * D, D), F._Fp8Heads(*out)
        c = F._RopeCs(*cs) if cs else None
        return L.gvr_fp8_quantize(ctypes.byref(xs), dtype, T, H, D, vp(pos), ctypes.byref(c) if c else None,
                                  ctypes.byref(os_), vp(slots), rows, flags, None)
    assert call(T=0) == 0 and call(H=0) == 0 and call(T=0, x=0, out=(0,) * 6, rows=0) == 0
    for kw in (dict(T=-1), dict(H=-1), dict(D=0), dict(D=-5), dict(dtype=3), dict(dtype=-1), dict(x=0), dict(x=257),
               dict(x=258, dtype=2), dict(out=(0, 256, 128, 1024, 2, 1)), dict(out=(512, 256, 128, 0, 2, 1)),
               dict(out=(512, 256, 128, 1026, 2, 1)), dict(slots=68), dict(rows=-1), dict(rows=3), dict(flags=2), dict(flags=4),
               dict(cs=(64, 10, 64, 0)), dict(cs=(64, 10, 256, 0), pos=64), dict(cs=(64, 10, 7, 0), pos=64),
               dict(cs=(64, 10, 64, F.kv4.ROPE_TRANSPOSED), pos=64), dict(cs=(0, 10, 64, 0), pos=64), dict(cs=(64, 10, 64, 0), pos=66)):
        assert call(**kw) == -1, kw
    for kw in (dict(T=1 << 31, rows=1 << 30), dict(rows=1 << 31), dict(H=(1 << 20) + 1), dict(D=(1 << 20) + 1),
               dict(H=1 << 20, D=1 << 15), dict(T=1 << 30, rows=1 << 30, H=1 << 14)):
        assert call(**kw) == -5, kw
    assert L.gvr_fp8_quantize(None, 0, 0, 1, 1, None, None, None, None, 0, 0, None) == -1


def test_quantize_matrix_checks(F):
    L = F.lib()

    def call(x=256, stride=300, dtype=0, R=5, C=300, a=(512, 300, 1024, 3, 1, 1, 0), b=None, flags=0):
        ms = [ctypes.byref(F._Fp8Matrix(*m)) if m else None for m in (a, b)]
        return L.gvr_fp8_quantize_matrix(vp(x), stride, dtype, R, C, ms[0], ms[1], flags, None)
    assert call(R=0) == 0 and call(C=0) == 0 and call(a=None) == 0 and call(R=0, x=0, a=(0, 0, 0, 0, 0, 1, 0)) == 0
    bad = (512, 300, 1024, 3, 1, 128, 0), (0, 300, 1024, 3, 1, 1, 0), (512, 300, 0, 3, 1, 1, 0), (512, 300, 1025, 3, 1, 1, 0), \
        (512, 300, 1024, 3, 1, 1, 1)
    for kw in [dict(a=m) for m in bad] + [dict(b=m) for m in bad] + [
            dict(R=-1), dict(C=-1), dict(dtype=3), dict(flags=4), dict(x=0), dict(x=257), dict(x=258, dtype=2), dict(flags=2)]:
        assert call(**kw) == -1, kw
    assert call(R=1 << 31) == -5 and call(C=1 << 31) == -5 and call(R=1 << 30, C=1 << 30) == -5


def test_matmul_checks(F):
    L = F.lib()
    A, B = (256, 300, 1024, 3, 1, 1, 0), (512, 300, 2048, 3, 1, 128, 0)

    def call(a=A, b=B, M=4, N=6, K=300, out=4096, dtype=0, ws=(None, 0)):
        return L.gvr_fp8_matmul(ctypes.byref(F._Fp8Matrix(*a)), ctypes.byref(F._Fp8Matrix(*b)), M, N, K, vp(out), N, dtype,
                                vp(ws[0]), ws[1], None)
    none = (0, 0, 0, 0, 0, 1, 0)
    assert call(M=0) == 0 and call(N=0) == 0 and call(M=0, a=none, b=none, out=0) == 0
    for kw in (dict(M=-1), dict(N=-1), dict(K=-1), dict(a=none), dict(b=none), dict(a=B), dict(b=B[:5] + (64, 0)),
               dict(a=A[:6] + (1,)), dict(a=(256, 300, 1026, 3, 1, 1, 0)), dict(out=0), dict(out=4097), dict(out=4098, dtype=2),
               dict(dtype=3), dict(ws=(None, 64)), dict(ws=(8, 64))):
        assert call(**kw) == -1, kw
    for kw in (dict(M=1 << 31), dict(N=1 << 31), dict(K=1 << 31), dict(M=1 << 30, N=1 << 30)):
        assert call(**kw) == -5, kw
    n = ctypes.c_size_t(7)
    a, b = ctypes.byref(F._Fp8Matrix(*A)), ctypes.byref(F._Fp8Matrix(*B))
    assert L.gvr_fp8_matmul_workspace(a, b, 4, 6, 300, None) == -1
    assert L.gvr_fp8_matmul_workspace(None, b, 4, 6, 300, ctypes.byref(n)) == -1
    assert L.gvr_fp8_matmul_workspace(b, a, 4, 6, 300, ctypes.byref(n)) == -1
    assert L.gvr_fp8_matmul_workspace(a, b, 0, 6, 300, ctypes.byref(n)) == 0 and n.value == 0


def test_page_step_checks(P):
    L = P.lib()

    def call(pool=None, args=None, ws=(64, 1 << 20)):
        p = dict(block_table=64, ctx_len=64, free_pages=64, free_count=64, width=4, pages=9, requests=3, page_size=16)
        a = dict(new_len=64, keep=None, T=8, ld=0, q_start=64, taken=64, positions=64, slots=64, dense=None, row_len=64)
        p.update(pool or {})
        a.update(args or {})
        return L.gvr_page_step(ctypes.byref(P._Pool(**p)), ctypes.byref(P._StepArgs(**a)), vp(ws[0]), ws[1], None)
    for kw in (dict(pool=dict(requests=-1)), dict(pool=dict(width=-1)), dict(pool=dict(pages=-1)), dict(pool=dict(page_size=0)),
               dict(pool=dict(page_size=48)), dict(pool=dict(page_size=1 << 17)), dict(pool=dict(block_table=0)),
               dict(pool=dict(ctx_len=0)), dict(pool=dict(free_pages=0)), dict(pool=dict(free_count=0)),
               dict(pool=dict(ctx_len=66)), dict(args=dict(T=-1)), dict(args=dict(new_len=0)), dict(args=dict(new_len=65)),
               dict(args=dict(slots=68)), dict(args=dict(dense=68)), dict(args=dict(dense=64, ld=-1)), dict(args=dict(keep=66)),
               dict(ws=(None, 0)), dict(ws=(72, 1 << 20))):
        assert call(**kw) == -1, kw
    for kw in (dict(pool=dict(requests=(1 << 20) + 1)), dict(pool=dict(width=1 << 28)), dict(pool=dict(pages=1 << 31)),
               dict(args=dict(T=1 << 31)), dict(args=dict(dense=64, ld=1 << 31))):
        assert call(**kw) == -5, kw
    assert call(ws=(64, int(L.gvr_page_step_workspace(3)) - 1)) == -3
    assert L.gvr_page_step_workspace(-1) == -1 and L.gvr_page_step_workspace((1 << 20) + 1) == -1
    assert L.gvr_page_step(None, None, None, 0, None) == -1
    with pytest.raises(ValueError):
        P.gvr_page_step_workspace(-3)


def test_binding_refuses(F, P):
    x = torch.zeros(2, 3, 128, dtype=torch.bfloat16)
    codes, scale = torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(4, 1)
    for f in (lambda: F.gvr_fp8_quantize(x), lambda: F.gvr_fp8_quantize(x[0]), lambda: F.gvr_fp8_quantize(x.int()),
              lambda: F.gvr_fp8_quantize_matrix(x[0]), lambda: F.gvr_fp8_quantize_matrix(x),
              lambda: F.gvr_fp8_matmul(codes, scale, codes, scale), lambda: F.gvr_fp8_linear(x, x[0]),
              lambda: F.gvr_fp8_matmul_workspace(codes, scale, codes, scale),
              lambda: P.gvr_page_step(P.new_page_pool(4, 16, 2, 3, device="cpu"), torch.zeros(2, dtype=torch.int32), 4),
              lambda: P.gvr_page_step((1, 2, 3, 4, 5), torch.zeros(2, dtype=torch.int32), 4)):
        with pytest.raises(ValueError):
            f()
