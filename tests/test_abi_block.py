"""Host-side checks of layer norm, rotary positions and attention: bad arguments are refused before a device is touched (no GPU, no compute call)."""
import ctypes as C
import os

import pytest

OK, NULL, SHAPE, DTYPE, ALIGN, ALIAS, WORKSPACE, UNSUPPORTED = range(8)
P = 0x100000                      # fake, aligned, never dereferenced: validation fails before any launch
F32, BF16 = 0, 1
BIG = 1 << 62


@pytest.fixture(scope="module")
def lib():
    from paper_2203_10991_amd import api
    if not os.path.exists(api.LIB_PATH):
        from paper_2203_10991_amd import build
        build.build()
    return api.load()


def test_layer_norm(lib):
    def fwd(x=P, ldx=32, xdt=BF16, w=P + 0x10000, b=P + 0x20000, wdt=F32, R=4, Cc=32, eps=1e-5, y=P + 0x30000, ldy=32, mean=P + 0x40000, rstd=P + 0x50000):
        return lib.nm_layer_norm(x, ldx, xdt, w, b, wdt, R, Cc, eps, y, ldy, mean, rstd, None)
    assert fwd(xdt=2) == DTYPE and fwd(wdt=-1) == DTYPE
    assert fwd(R=-1) == SHAPE and fwd(Cc=0) == SHAPE and fwd(Cc=32769, ldx=1 << 20, ldy=1 << 20) == SHAPE and b"32768" in lib.nm_last_error()
    assert fwd(ldx=31) == SHAPE and fwd(ldy=31) == SHAPE and fwd(R=BIG, ldx=BIG) == SHAPE
    assert fwd(x=None) == NULL and fwd(y=None) == NULL
    assert fwd(x=P + 1) == ALIGN and fwd(y=P + 0x30001) == ALIGN and fwd(w=P + 0x10002) == ALIGN and fwd(b=P + 0x20001, wdt=BF16) == ALIGN and fwd(mean=P + 0x40002) == ALIGN
    assert fwd(y=P) == ALIAS and fwd(y=P + 0x10000) == ALIAS and fwd(mean=P) == ALIAS and fwd(rstd=P + 0x40000) == ALIAS and fwd(mean=P + 0x30000) == ALIAS and fwd(rstd=P + 0x20000) == ALIAS
    assert fwd(eps=-1.0) == UNSUPPORTED and fwd(eps=float("inf")) == UNSUPPORTED and fwd(eps=float("nan")) == UNSUPPORTED
    assert fwd(R=0) == OK and lib.nm_last_error() == b""

    need = lib.nm_layer_norm_grad_workspace(4, 32)

    def grad(g=P, x=P + 0x10000, ld=32, xdt=BF16, w=P + 0x20000, wdt=F32, mean=P + 0x30000, rstd=P + 0x40000, R=4, dx=P + 0x50000, dw=P + 0x60000, db=P + 0x70000, ws=P + 0x80000, n=need):
        return lib.nm_layer_norm_grad(g, ld, x, ld, xdt, w, wdt, mean, rstd, R, 32, dx, ld, dw, db, ws, n, None)
    assert need >= 256 and lib.nm_layer_norm_grad_workspace(0, 32) == 0 and lib.nm_layer_norm_grad_workspace(4, 0) == 0 and lib.nm_layer_norm_grad_workspace(4, 32769) == 0
    assert grad(ws=None) == WORKSPACE and grad(n=need - 1) == WORKSPACE and grad(ws=P + 0x80004) == ALIGN
    assert grad(mean=None) == NULL and grad(rstd=None) == NULL and grad(g=None) == NULL and grad(dx=None) == NULL
    assert grad(dw=P + 0x60002) == ALIGN and grad(db=P + 0x70001) == ALIGN
    assert grad(dx=P) == ALIAS and grad(dx=P + 0x10000) == ALIAS and grad(dw=P + 0x20000) == ALIAS and grad(db=P + 0x60000) == ALIAS and grad(ws=P + 0x50000) == ALIAS and grad(ws=P + 0x30000) == ALIAS
    assert grad(xdt=7) == DTYPE and grad(ld=30) == SHAPE and grad(R=-1) == SHAPE


def _heads(data=P, batch=1 << 12, token=64, head=32):
    from paper_2203_10991_amd.api import _Heads
    return C.byref(_Heads(data, batch, token, head))


def test_rotary(lib):
    def call(x=None, y=None, dt=BF16, B=2, T=4, H=2, D=32, part=16, freqs=P + 0x200000, pos=P + 0x300000, bits=64, stride=4, scale=1.0):
        return lib.nm_rotary(_heads() if x is None else x, _heads(P + 0x100000) if y is None else y, dt, B, T, H, D, part, freqs, pos, bits, stride, 0, scale, 0, None)
    assert call(dt=3) == DTYPE and call(bits=16) == DTYPE
    assert call(B=-1) == SHAPE and call(D=1) == SHAPE and call(D=1026) == SHAPE and call(part=0) == SHAPE and call(part=15) == SHAPE and call(part=34) == SHAPE
    assert call(B=1 << 20, T=1 << 20) == SHAPE and call(stride=-1) == SHAPE and call(x=_heads(token=-64)) == SHAPE and call(x=_heads(batch=BIG)) == SHAPE
    assert call(y=_heads(P + 0x100000, head=0)) == SHAPE and call(y=_heads(P + 0x100000, token=0)) == SHAPE and call(y=_heads(P + 0x100000, token=48)) == SHAPE   # elements that share memory
    assert call(freqs=None) == NULL and call(x=_heads(None)) == NULL and call(y=_heads(None)) == NULL
    assert call(freqs=P + 4) == ALIGN and call(pos=P + 0x300004) == ALIGN and call(x=_heads(P + 1)) == ALIGN
    assert call(y=_heads(P + 2)) == ALIAS and call(y=_heads(P, head=64, token=128)) == ALIAS and call(freqs=P + 0x100000) == ALIAS and call(pos=P + 0x100000) == ALIAS
    assert call(scale=float("inf")) == UNSUPPORTED
    assert call(B=0) == OK and call(T=0, freqs=None) == OK and lib.nm_last_error() == b""


def test_attention(lib):
    def tensor(i, **kw):
        return _heads(P + i * 0x100000, **{**dict(batch=1 << 14, token=64, head=32), **kw})

    def sizes(B=2, Tq=8, Tk=8, Hq=2, Hk=2, D=32, dt=BF16):
        return B, Tq, Tk, Hq, Hk, D, dt

    def fwd(q=tensor(0), k=tensor(1), v=tensor(2), o=tensor(3), lse=P + 0x400000, rest=None, scale=0.5, ql=None, kl=None, ws=None, n=0, **kw):
        return lib.nm_attention(q, k, v, o, lse, rest, *sizes(**kw), 0, scale, ql, kl, ws, n, None)
    assert fwd(dt=2) == DTYPE
    for bad in (dict(B=-1), dict(Tq=-1), dict(D=4), dict(D=12), dict(D=136), dict(Hq=3), dict(Hq=0), dict(Hk=0), dict(Hq=1), dict(Tk=1 << 31), dict(Tq=1 << 30, Hq=4), dict(B=1 << 40)):
        assert fwd(**bad) == SHAPE, bad
    assert fwd(q=tensor(0, token=-64)) == SHAPE and fwd(o=tensor(3, head=0)) == SHAPE and fwd(o=tensor(3, token=32)) == SHAPE
    assert fwd(q=None) == NULL and fwd(q=_heads(None)) == NULL and fwd(o=_heads(None)) == NULL
    assert fwd(q=_heads(P + 8)) == ALIGN and fwd(k=tensor(1, token=65)) == ALIGN and fwd(k=tensor(1, token=66), dt=F32) == ALIGN and fwd(o=tensor(3, head=36)) == ALIGN
    assert fwd(lse=P + 0x400002) == ALIGN and fwd(rest=P + 0x480002) == ALIGN and fwd(rest=P) == ALIAS and fwd(rest=P + 0x400000) == ALIAS and fwd(ql=P + 2) == ALIGN and fwd(kl=P + 1) == ALIGN
    assert fwd(o=tensor(0)) == ALIAS and fwd(o=tensor(2)) == ALIAS and fwd(lse=P) == ALIAS and fwd(lse=P + 0x300000) == ALIAS and fwd(kl=P + 0x300000) == ALIAS
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert fwd(scale=scale) == UNSUPPORTED
    need = lib.nm_attention_workspace(*sizes(Tq=1, Tk=100000))
    assert need > 0 and lib.nm_attention_workspace(*sizes(D=12)) == 0 and lib.nm_attention_workspace(*sizes(B=0)) == 0
    far = dict(k=tensor(0x10, batch=1 << 24), v=tensor(0x1000, batch=1 << 24), Tq=1, Tk=100000, lse=None)
    assert fwd(**far) == WORKSPACE and fwd(**far, ws=P + 0x500000, n=need - 1) == WORKSPACE and fwd(**far, ws=P + 0x500004, n=need) == ALIGN and fwd(**far, ws=P + 0x300000, n=need) == ALIAS
    assert fwd(B=0) == OK and fwd(Tq=0, o=_heads(None)) == OK and lib.nm_last_error() == b""

    need = lib.nm_attention_grad_workspace(*sizes())
    assert need >= 2 * 2 * 8 * 4 and lib.nm_attention_grad_workspace(*sizes(Tq=0)) == 0

    def grad(g=tensor(0), q=tensor(1), k=tensor(2), v=tensor(3), o=tensor(4), lse=P + 0x500000, rest=P + 0x580000, dq=tensor(6), dk=tensor(7), dv=tensor(8), ws=P + 0x900000, n=need, **kw):
        return lib.nm_attention_grad(g, q, k, v, o, lse, rest, *sizes(**kw), 0, 0.5, None, None, dq, dk, dv, ws, n, None)
    assert grad(lse=None) == NULL and grad(rest=P + 0x580001) == ALIGN and grad(rest=P + 0x600000) == ALIAS and grad(dk=None) == NULL and grad(dv=_heads(None)) == NULL and grad(g=_heads(None)) == NULL
    assert grad(ws=None) == WORKSPACE and grad(n=need - 1) == WORKSPACE and grad(ws=P + 0x900008) == ALIGN
    assert grad(dq=tensor(0)) == ALIAS and grad(dk=tensor(6)) == ALIAS and grad(dv=tensor(4)) == ALIAS and grad(ws=P + 0x600000) == ALIAS and grad(ws=P + 0x500000) == ALIAS
    assert grad(dq=tensor(6, head=0)) == SHAPE and grad(Hq=3) == SHAPE
    # parts of one tensor side by side are no overlap, shifted ones are
    base = P + 0x600000
    parts = lambda step: [_heads(base + i * step, 19200, 192, 32) for i in range(3)]       # noqa: E731
    inside = parts(128 - 16)
    assert grad(dq=inside[0], dk=inside[1], dv=inside[2]) == ALIAS
    whole = parts(128)
    assert grad(dq=whole[0], dk=whole[1], dv=whole[2], n=0) == WORKSPACE
    assert grad(dq=whole[0], dk=whole[1], dv=_heads(base + 256 + 16, 19200, 192, 32), n=need) == ALIAS
