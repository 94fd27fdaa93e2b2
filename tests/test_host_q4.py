"""Refusals of the 4-bit weights' entry points and of the norm that need no GPU: argument checks come before any device work."""
import ctypes

import pytest
import torch

F32, F16, BF16, I8 = range(4)
NULL, SHAPE, MISMATCH, UNSUPPORTED, DEVICE, HANDLE = 1, 2, 3, 4, 6, 7
ll, fl = ctypes.c_longlong, ctypes.c_float


@pytest.fixture(scope="module")
def L():
    import os
    from paper_2212_08815_amd import fscnn
    if not os.path.exists(fscnn.LIB_PATH):
        from paper_2212_08815_amd import build
        build.build()
    return fscnn.lib()


fake, odd = ctypes.c_void_p(256), ctypes.c_void_p(257)


def test_weights(L):
    h = ctypes.c_void_p()
    ref = ctypes.byref(h)
    comp = lambda w=fake, t=F32, K=4, C=8, ld=8, g=128, z=0, out=ref: L.fscnn_q4_compress(w, t, K, C, ll(ld), g, z, None, out)
    imp = lambda c=fake, s=fake, t=F16, z=None, K=4, C=8, g=128, out=ref: L.fscnn_q4_import(c, s, t, z, K, C, g, None, out)
    assert comp(w=None) == comp(out=None) == imp(c=None) == imp(s=None) == imp(out=None) == NULL
    for t in (I8, 4, -1, 1 << 30):
        assert comp(t=t) == imp(t=t) == UNSUPPORTED
    assert imp(t=F32) == UNSUPPORTED                       # scales are 16 bits
    for K, C in ((0, 8), (4, 0), (-1, 8), (4, -5)):
        assert comp(K=K, C=C) == imp(K=K, C=C) == SHAPE
    assert comp(ld=7) == comp(ld=-8) == comp(ld=1 << 40) == SHAPE
    for g in (0, 16, 33, 256, -32):
        assert comp(g=g) == imp(g=g) == UNSUPPORTED
    assert comp(C=(1 << 20) + 1, ld=1 << 21) == imp(C=(1 << 20) + 1) == UNSUPPORTED
    assert comp(w=odd) == imp(s=odd) == UNSUPPORTED
    junk = (ctypes.c_ubyte * 512)()
    jp = ctypes.byref(junk)
    assert L.fscnn_q4_info(None, None, None, None, None, None) == NULL and L.fscnn_q4_info(jp, None, None, None, None, None) == HANDLE
    assert L.fscnn_q4_export(None, fake, fake, None) == L.fscnn_q4_export(jp, None, fake, None) == L.fscnn_q4_export(jp, fake, None, None) == NULL
    assert L.fscnn_q4_export(jp, fake, fake, None) == HANDLE
    assert L.fscnn_q4_destroy(None) == NULL and L.fscnn_q4_destroy(jp) == HANDLE
    if not torch.cuda.is_available():
        assert comp() == imp() == DEVICE
    assert not h.value


def test_linear(L):
    junk = (ctypes.c_ubyte * 512)()
    jp = ctypes.byref(junk)
    lin = lambda q=jp, x=fake, M=1: L.fscnn_linear_q4(q, x, F32, ll(8), None, 1, M, 8, None, fl(1), ctypes.c_void_p(512), F32, ll(8), None, ll(0), None)
    assert lin(q=None) == lin(x=None) == NULL
    assert lin() == lin(M=0) == lin(M=-1) == HANDLE
    assert L.fscnn_linear_q4_workspace(None, F32, 1) == L.fscnn_linear_q4_workspace(jp, F32, 1) == -1


def test_norm(L):
    other, third = ctypes.c_void_p(1 << 20), ctypes.c_void_p(1 << 21)

    def norm(x=fake, t=BF16, ldx=8, r=None, ldr=8, ro=None, ldo=8, w=None, wt=F32, M=2, D=8, eps=1e-6, y=other, yt=BF16, ldy=8, s=None, g=0):
        return L.fscnn_rms_norm(x, t, ll(ldx), r, ll(ldr), ro, ll(ldo), w, wt, M, D, fl(eps), y, yt, ll(ldy), s, g, None)

    assert norm(x=None) == norm(y=None) == norm(yt=I8, s=None) == NULL
    assert norm(M=-1) == norm(D=0) == norm(D=-3) == norm(eps=-1.0) == norm(eps=float("nan")) == SHAPE
    assert norm(ldx=7) == norm(ldy=7) == norm(r=third, ldr=7) == norm(r=third, ro=ctypes.c_void_p(1 << 22), ldo=0) == SHAPE
    assert norm(ldx=1 << 62) == SHAPE
    for t in (I8, 4, -1):
        assert norm(t=t) == norm(w=fake, wt=t) == UNSUPPORTED
    assert norm(yt=4) == norm(yt=-1) == norm(D=65537, ldx=70000, ldy=70000) == UNSUPPORTED
    for g in (16, 100, 256, -32):
        assert norm(yt=I8, s=third, g=g) == UNSUPPORTED
    assert norm(g=32) == norm(s=third) == UNSUPPORTED      # scales belong to an 8-bit output
    assert norm(ro=third) == UNSUPPORTED                   # no sum without a residual
    assert norm(x=odd) == norm(y=odd) == norm(r=odd) == norm(w=odd) == norm(r=third, ro=odd) == norm(yt=I8, s=odd) == UNSUPPORTED
    # in place: the same type and row distance only, and not both outputs
    assert norm(y=fake, yt=F16) == norm(y=fake, yt=I8, s=third) == norm(y=fake, ldy=9) == UNSUPPORTED
    assert norm(r=third, y=third, yt=F32) == norm(r=third, y=third, ldy=9) == UNSUPPORTED
    assert norm(r=third, ro=third, ldo=9) == norm(r=third, ro=fake, ldo=9) == norm(r=third, ro=other) == UNSUPPORTED
    assert norm(M=0) == norm(M=0, x=None, y=None) == norm(M=0, yt=I8) == 0
    if not torch.cuda.is_available():
        assert norm() == norm(r=third, ro=third) == norm(y=fake) == norm(w=fake, wt=F16) == norm(yt=I8, s=third, g=64) == DEVICE


def test_binding_refuses_what_is_not_on_the_gpu():
    from paper_2212_08815_amd import fscnn
    z = torch.zeros(4, 8)
    for call in (lambda: fscnn.q4_compress(z), lambda: fscnn.q4_import(z.byte(), z.half()), lambda: fscnn.rms_norm(z), lambda: fscnn.rms_norm_q8(z),
                 lambda: fscnn.rms_norm(None)):
        with pytest.raises(TypeError):
            call()


def test_native_calls_count_and_read_their_arguments(L):
    from paper_2212_08815_amd import fscnn
    m = fscnn._native()
    junk = (ctypes.c_ubyte * 512)()
    h = ctypes.addressof(junk)
    args = [h, 256, F32, 8, None, 1, 1, 8, None, 1.0, 512, F32, 8, None, 0, 0]
    assert m.linear_q4(*args) == HANDLE
    for i, v, err in ((3, "8", TypeError), (3, 1 << 70, OverflowError), (6, 1 << 31, OverflowError), (9, "x", TypeError), (2, None, TypeError)):
        with pytest.raises(err):
            m.linear_q4(*(args[:i] + [v] + args[i + 1:]))
    with pytest.raises(TypeError):
        m.linear_q4(*args[:-1])
    with pytest.raises(TypeError):
        m.rms_norm(*args)
    norm = [None, BF16, 8, None, 0, None, 0, None, F32, 0, 8, 1e-6, None, BF16, 8, None, 0, 0]
    assert m.rms_norm(*norm) == 0
    with pytest.raises(TypeError):
        m.rms_norm(*(norm[:11] + [None] + norm[12:]))
