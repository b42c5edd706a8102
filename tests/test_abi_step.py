"""Host-side checks of the entry points around the update phase -- 8-bit integer products, embedding, AdamW: bad arguments are refused before a device is touched
(no GPU, no compute call)."""
import ctypes as C
import os

import pytest

OK, NULL, SHAPE, DTYPE, ALIGN, ALIAS, WORKSPACE, UNSUPPORTED = range(8)
P = 0x10000                       # fake, aligned, never dereferenced: validation fails before any launch
F32, BF16 = 0, 1
BIG = 1 << 62


@pytest.fixture(scope="module")
def lib():
    from paper_2203_10991_amd import api
    if not os.path.exists(api.LIB_PATH):
        from paper_2203_10991_amd import build
        build.build()
    return api.load()


def test_quantisers(lib):
    def rows(x=P, R=4, C=32, ldx=32, dt=BF16, q=P + 0x10000, ldq=32, scale=P + 0x20000):
        return lib.nm_quant_i8(x, R, C, ldx, dt, q, ldq, scale, None)
    assert rows(dt=2) == DTYPE
    assert rows(R=-1) == SHAPE and rows(C=-1) == SHAPE and rows(ldx=16) == SHAPE and rows(R=BIG, ldx=BIG) == SHAPE
    assert rows(ldq=16) == SHAPE and rows(ldq=40) == ALIGN and rows(ldq=1 << 22) == SHAPE
    assert rows(x=None) == NULL and rows(q=None) == NULL and rows(scale=None) == NULL
    assert rows(x=P + 1) == ALIGN and rows(q=P + 8) == ALIGN and rows(scale=P + 2) == ALIGN
    assert rows(q=P) == ALIAS and rows(scale=P + 0x10000) == ALIAS and rows(scale=P) == ALIAS
    assert rows(R=0) == OK and lib.nm_last_error() == b""

    def cols(ws=P + 0x30000, bytes=None, C=32, q=P + 0x10000, ldq=16):
        need = lib.nm_quant_i8_t_workspace(4, C)
        return lib.nm_quant_i8_t(P, 4, C, 32, BF16, q, ldq, P + 0x20000, ws, need if bytes is None else bytes, None)
    assert lib.nm_quant_i8_t_workspace(4, 32) >= 128 and lib.nm_quant_i8_t_workspace(-1, 32) == 0 and lib.nm_quant_i8_t_workspace(4, 0) == 0
    assert cols(ws=None) == WORKSPACE and cols(bytes=0) == WORKSPACE and cols(ws=P + 0x30004) == ALIGN
    assert cols(ws=P) == ALIAS and cols(ws=P + 0x10000) == ALIAS and cols(ws=P + 0x20000) == ALIAS and cols(q=P) == ALIAS
    assert cols(ldq=8) == ALIGN


def test_products(lib):
    def gemm(xq=P, ldx=64, xs=P + 0x10000, wq=P + 0x20000, ldw=64, ws=P + 0x30000, bias=P + 0x40000, bdt=F32, T=4, O=8, I=50, y=P + 0x50000, ldy=8, ydt=BF16):
        return lib.nm_gemm_i8(xq, ldx, xs, wq, ldw, ws, bias, bdt, T, O, I, 0, y, ldy, ydt, None)
    assert gemm(I=0) == SHAPE and b"131072" in lib.nm_last_error()
    assert gemm(I=131073, ldx=1 << 18, ldw=1 << 18) == SHAPE and gemm(T=-1) == SHAPE and gemm(O=-1) == SHAPE and gemm(T=BIG) == SHAPE
    assert gemm(ldx=48) == SHAPE and gemm(ldw=60) == ALIGN and gemm(ldx=72) == ALIGN and gemm(ldw=1 << 22) == SHAPE and gemm(ldy=1 << 22) == SHAPE and gemm(ldy=7) == SHAPE
    assert gemm(xq=None) == NULL and gemm(xs=None) == NULL and gemm(wq=None) == NULL and gemm(ws=None) == NULL and gemm(y=None) == NULL
    assert gemm(ydt=3) == DTYPE and gemm(bdt=7) == DTYPE
    assert gemm(xq=P + 8) == ALIGN and gemm(wq=P + 0x20004) == ALIGN and gemm(y=P + 0x50001) == ALIGN and gemm(bias=P + 0x40002) == ALIGN and gemm(bias=P + 0x40001, bdt=BF16) == ALIGN
    assert gemm(y=P) == ALIAS and gemm(y=P + 0x10000) == ALIAS and gemm(y=P + 0x20000) == ALIAS and gemm(y=P + 0x30000) == ALIAS and gemm(y=P + 0x40000) == ALIAS
    assert gemm(T=0) == OK and gemm(O=0) == OK and lib.nm_last_error() == b""

    def linear(x=P, ldx=50, xdt=F32, ws=P + 0x60000, bytes=None, y=P + 0x50000, T=4, I=50, bias=None):
        need = lib.nm_linear_i8_workspace(4, 50)
        return lib.nm_linear_i8(x, ldx, xdt, P + 0x20000, 64, P + 0x30000, bias, 0, T, 8, I, 1, y, 8, F32, ws, need if bytes is None else bytes, None)
    assert lib.nm_linear_i8_workspace(4, 50) == 4 * 128 + 16 and lib.nm_linear_i8_workspace(0, 50) == 0 and lib.nm_linear_i8_workspace(4, 131073) == 0
    assert linear(ws=None) == WORKSPACE and linear(bytes=100) == WORKSPACE and linear(ws=P + 0x60008) == ALIGN
    assert linear(x=None) == NULL and linear(xdt=2) == DTYPE and linear(ldx=49) == SHAPE and linear(x=P + 2) == ALIGN
    assert linear(y=P) == ALIAS and linear(ws=P) == ALIAS and linear(ws=P + 0x20000) == ALIAS and linear(ws=P + 0x30000) == ALIAS and linear(ws=P + 0x50000) == ALIAS
    assert linear(T=0) == OK


def test_embedding(lib):
    def look(table=P, V=10, D=16, ldt=16, tdt=BF16, ids=P + 0x10000, bits=64, N=5, out=P + 0x20000, ldo=16, odt=F32):
        return lib.nm_embed(table, V, D, ldt, tdt, ids, bits, N, 1.0, out, ldo, odt, None)
    assert look(tdt=2) == DTYPE and look(odt=-1) == DTYPE and look(bits=16) == DTYPE
    assert look(N=-1) == SHAPE and look(N=1 << 31) == SHAPE and look(V=-1) == SHAPE and look(ldt=15) == SHAPE and look(ldo=15) == SHAPE and look(V=BIG, ldt=BIG) == SHAPE
    assert look(table=None) == NULL and look(ids=None) == NULL and look(out=None) == NULL
    assert look(table=P + 1) == ALIGN and look(ids=P + 0x10004) == ALIGN and look(out=P + 0x20002) == ALIGN
    assert look(out=P) == ALIAS and look(out=P + 0x10000) == ALIAS
    assert look(N=0) == OK and look(D=0) == OK

    def grad(g=P, ldg=16, ids=P + 0x10000, N=5, V=10, D=16, out=P + 0x20000, ldo=16, ws=P + 0x40000, bytes=None):
        need = lib.nm_embed_grad_workspace(5, 10, 16)
        return lib.nm_embed_grad(g, ldg, BF16, ids, 32, N, V, D, 1.0, -1, 0, out, ldo, F32, ws, need if bytes is None else bytes, None)
    assert lib.nm_embed_grad_workspace(5, 10, 16) > 0 and lib.nm_embed_grad_workspace(0, 10, 16) == 0 and lib.nm_embed_grad_workspace(5, 1 << 31, 16) == 0
    assert grad(ws=None) == WORKSPACE and grad(bytes=16) == WORKSPACE and grad(ws=P + 0x40008) == ALIGN
    assert grad(g=None) == NULL and grad(out=None) == NULL and grad(V=1 << 31) == SHAPE and grad(ldg=8) == SHAPE and grad(ldo=8) == SHAPE
    assert grad(out=P) == ALIAS and grad(out=P + 0x10000) == ALIAS and grad(ws=P) == ALIAS and grad(ws=P + 0x10000) == ALIAS and grad(ws=P + 0x20000) == ALIAS
    assert grad(V=0) == OK and grad(D=0) == OK


def test_adamw(lib):
    from paper_2203_10991_amd.api import _AdamwTensor

    def step(count=1, pt=F32, gt=F32, state=0, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, wd=0.0, step=1, tensors=None, dev=None, **kw):
        a = dict(param=P, grad=P + 0x10000, m=P + 0x20000, v=P + 0x30000, m_scale=P + 0x40000, v_scale=P + 0x50000, master=None, n=8, number=0)
        a.update(kw)
        t = (_AdamwTensor * 1)(_AdamwTensor(*a.values())) if tensors is None else tensors
        return lib.nm_adamw(t, count, pt, gt, state, lr, b1, b2, eps, wd, step, 1.0, dev, 0, None)
    assert step(pt=2) == DTYPE and step(gt=5) == DTYPE and step(state=2) == UNSUPPORTED
    assert step(count=-1) == SHAPE and step(step=0) == SHAPE and step(step=1 << 31) == SHAPE and step(n=-1) == SHAPE and step(n=1 << 41) == SHAPE
    assert step(b1=1.0) == UNSUPPORTED and step(b2=-0.1) == UNSUPPORTED and step(b1=float("nan")) == UNSUPPORTED
    assert step(eps=-1.0) == UNSUPPORTED and step(eps=float("inf")) == UNSUPPORTED and step(lr=float("nan")) == UNSUPPORTED and step(wd=float("inf")) == UNSUPPORTED
    for k in ("param", "grad", "m", "v"):
        assert step(**{k: None}) == NULL
    assert step(state=1, m_scale=None) == NULL and step(state=1, v_scale=None) == NULL
    assert step(param=P + 2) == ALIGN and step(grad=P + 0x10001, gt=BF16) == ALIGN and step(m=P + 0x20002) == ALIGN and step(state=1, m_scale=P + 0x40001) == ALIGN and step(dev=P + 1) == ALIGN
    assert step(master=P + 0x60000) == UNSUPPORTED
    assert step(grad=P) == ALIAS and step(v=P + 0x20000) == ALIAS and step(state=1, v_scale=P + 0x40000) == ALIAS and step(pt=BF16, master=P + 0x30000) == ALIAS
    two = (_AdamwTensor * 2)(_AdamwTensor(P, P + 0x10000, P + 0x20000, P + 0x30000, None, None, P + 0x60000, 8, 0),
                             _AdamwTensor(P + 0x70000, P + 0x80000, P + 0x90000, P + 0xa0000, None, None, None, 8, 1))
    assert step(count=2, pt=BF16, tensors=two) == UNSUPPORTED and b"two calls" in lib.nm_last_error()
    assert step(count=0) == OK and step(n=0, param=None) == OK and lib.nm_last_error() == b""
    assert lib.nm_adamw(None, 1, 0, 0, 0, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1, 1.0, None, 0, None) == NULL
