"""Refusals of the gradient operators' entry points: every bad argument is answered on the host before anything is
queued.  No GPU is used: the pointers below are never dereferenced."""
import ctypes

import pytest

import paper_2607_19331_amd as iso
from paper_2607_19331_amd import _lib

FAKE = 0x100000
WS = FAKE * 16


def embed(**kw):
    a = dict(ids=FAKE, tokens=8, vocab=64, dim=16, x=FAKE, table=FAKE, grad=FAKE, id_type=_lib.I64)
    a.update(kw)
    return iso.Embed(**a)


def lookup(e, dt=iso.BF16, ws=WS, ws_bytes=1 << 30):
    return _lib.load().iso_embed_lookup(ctypes.byref(iso._embed(e)), dt, ws, ws_bytes, None)


def grad(e, dt=iso.BF16, dtg=iso.F32, acc=0, ws=WS, ws_bytes=1 << 30):
    return _lib.load().iso_embed_grad(ctypes.byref(iso._embed(e)), dt, dtg, acc, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [lookup, grad])
def test_embed_refusals(call):
    assert call(embed(tokens=-1)) == _lib.ERR_INVALID_ARG
    assert call(embed(vocab=0)) == _lib.ERR_INVALID_ARG
    assert call(embed(dim=0)) == _lib.ERR_INVALID_ARG
    assert call(embed(id_type=2)) == _lib.ERR_INVALID_ARG
    assert call(embed(ids=None)) == _lib.ERR_INVALID_ARG
    assert call(embed(x=None)) == _lib.ERR_INVALID_ARG
    assert call(embed(ld_x=15)) == _lib.ERR_INVALID_ARG
    assert call(embed(scale=float("nan"))) == _lib.ERR_INVALID_ARG
    assert call(embed(scale=1e300)) == _lib.ERR_INVALID_ARG
    assert call(embed(), dt=2) == _lib.ERR_INVALID_ARG
    assert call(embed(table=None, grad=None)) == _lib.ERR_INVALID_ARG
    assert call(embed(ids=FAKE + 4)) == _lib.ERR_ALIGNMENT
    assert call(embed(x=FAKE + 8)) == _lib.ERR_ALIGNMENT
    assert call(embed(table=FAKE + 2, grad=FAKE + 2)) == _lib.ERR_ALIGNMENT
    assert call(embed(), ws=WS + 64) == _lib.ERR_ALIGNMENT
    assert call(embed(), ws=None) == _lib.ERR_WORKSPACE
    assert call(embed(), ws_bytes=255) == _lib.ERR_WORKSPACE
    assert call(embed(tokens=1 << 31)) == _lib.ERR_UNSUPPORTED
    assert call(embed(vocab=_lib.EMBED_MAX_VOCAB + 1)) == _lib.ERR_UNSUPPORTED
    assert call(embed(dim=(1 << 18) + 1)) == _lib.ERR_UNSUPPORTED
    assert call(embed(tokens=1 << 30, ld_x=1 << 30)) == _lib.ERR_UNSUPPORTED
    # an id pointer of its own size is enough; the workspace is checked last
    assert call(embed(ids=FAKE + 4, id_type=_lib.I32), ws_bytes=16) == _lib.ERR_WORKSPACE


def test_embed_more_refusals():
    L = _lib.load()
    assert L.iso_embed_lookup(None, iso.BF16, WS, 1 << 30, None) == _lib.ERR_INVALID_ARG
    assert L.iso_embed_grad(None, iso.BF16, iso.F32, 0, WS, 1 << 30, None) == _lib.ERR_INVALID_ARG
    assert grad(embed(), dtg=7) == _lib.ERR_INVALID_ARG
    assert grad(embed(), acc=2) == _lib.ERR_INVALID_ARG
    for n in (8, 10000):
        need = L.iso_workspace_size_embed(ctypes.byref(iso._embed(embed(tokens=n))))
        assert need >= 256 and grad(embed(tokens=n), ws_bytes=need - 1) == _lib.ERR_WORKSPACE
    assert need > 10000 * 4
    assert L.iso_workspace_size_embed(None) == 0
    assert L.iso_workspace_size_embed(ctypes.byref(iso._embed(embed(vocab=-3)))) == 0
    with pytest.raises(TypeError):
        iso._embed(embed(id_type=None))
    with pytest.raises(ValueError):
        iso.embed_workspace(embed(dim=0), "cpu")


def ckpt(**kw):
    a = dict(rows=4, cols=40, q=FAKE, e=FAKE, x=FAKE)
    a.update(kw)
    return iso.Ckpt(**a)


def table(call, cs, dt=iso.F32, n=None):
    arr = (_lib.IsoCkpt * max(1, len(cs)))(*[iso._ckpt(c) for c in cs])
    return getattr(_lib.load(), call)(arr, len(cs) if n is None else n, dt, None)


@pytest.mark.parametrize("call", ["iso_ckpt_pack", "iso_ckpt_unpack"])
def test_ckpt_refusals(call):
    ok = ckpt(rows=0)
    assert table(call, [ok, ckpt(rows=-1)]) == _lib.ERR_INVALID_ARG
    assert table(call, [ok, ckpt(cols=-1)]) == _lib.ERR_INVALID_ARG
    assert table(call, [ckpt(q=None)]) == _lib.ERR_INVALID_ARG
    assert table(call, [ckpt(e=None)]) == _lib.ERR_INVALID_ARG
    assert table(call, [ckpt(x=None)]) == _lib.ERR_INVALID_ARG
    assert table(call, [ckpt(ld_x=39)]) == _lib.ERR_INVALID_ARG
    assert table(call, [ckpt()], dt=-1) == _lib.ERR_INVALID_ARG
    assert table(call, [ckpt()], n=-1) == _lib.ERR_INVALID_ARG
    assert getattr(_lib.load(), call)(None, 1, iso.F32, None) == _lib.ERR_INVALID_ARG
    assert table(call, [ckpt(q=FAKE + 8)]) == _lib.ERR_ALIGNMENT
    assert table(call, [ckpt(e=FAKE + 1)]) == _lib.ERR_ALIGNMENT
    assert table(call, [ckpt(x=FAKE + 4)]) == _lib.ERR_ALIGNMENT
    assert table(call, [ckpt(cols=(1 << 24) + 1)]) == _lib.ERR_UNSUPPORTED
    assert table(call, [ckpt(rows=1 << 40)]) == _lib.ERR_UNSUPPORTED
    assert table(call, [ckpt(ld_x=1 << 62)]) == _lib.ERR_UNSUPPORTED
    with pytest.raises(iso.IsoError, match="invalid argument"):
        getattr(iso, call)([ckpt(q=None)], iso.F32, stream=0)


def test_ckpt_ld():
    assert [iso.iso_ckpt_ld(c) for c in (0, 1, 31, 32, 33, 18944)] == [0, 32, 32, 32, 64, 18944]
    assert iso.iso_ckpt_ld(-1) == -1 and iso.iso_ckpt_ld((1 << 63) - 1) == -1
    q, e = iso.ckpt_buffers(3, 33, "cpu")
    assert tuple(q.shape) == (3, 64) and tuple(e.shape) == (3, 2)


def gate(gk={}, uk={}, dt=iso.BF16, **kw):
    a = dict(dh=FAKE, dgate=FAKE, dup=FAKE)
    a.update(kw)
    g = iso.GateGrad(ckpt(**gk), ckpt(**uk), **a)
    arr = (_lib.IsoGateGrad * 1)(_lib.IsoGateGrad(iso._ckpt(g.gate), iso._ckpt(g.up), g.dh, g.dgate, g.dup,
                                                  g.gate.cols if g.ld is None else g.ld))
    return _lib.load().iso_ckpt_gate_grad(arr, 1, dt, None)


def test_gate_refusals():
    assert gate(gk=dict(rows=5)) == _lib.ERR_INVALID_ARG
    assert gate(uk=dict(cols=41)) == _lib.ERR_INVALID_ARG
    assert gate(gk=dict(q=None)) == _lib.ERR_INVALID_ARG
    assert gate(uk=dict(e=FAKE + 1)) == _lib.ERR_ALIGNMENT
    assert gate(dh=None) == _lib.ERR_INVALID_ARG
    assert gate(dgate=None) == _lib.ERR_INVALID_ARG
    assert gate(dup=FAKE + 2) == _lib.ERR_ALIGNMENT
    assert gate(ld=39) == _lib.ERR_INVALID_ARG
    assert gate(ld=1 << 62) == _lib.ERR_UNSUPPORTED
    assert gate(dt=5) == _lib.ERR_INVALID_ARG
    assert _lib.load().iso_ckpt_gate_grad(None, 1, iso.BF16, None) == _lib.ERR_INVALID_ARG


def layer(ck={}, **kw):
    a = dict(dy=FAKE, grad=FAKE, rows=24)
    a.update(kw)
    return iso.WeightGrad(ckpt(**ck), **a)


def wgrad(js, dt=iso.BF16, dtg=iso.F32, acc=0, ws=WS, ws_bytes=1 << 40):
    return _lib.load().iso_ckpt_weight_grad(iso._weight_grads(js), len(js), dt, dtg, acc, ws, ws_bytes, None)


def test_weight_grad_refusals():
    L = _lib.load()
    assert wgrad([layer(rows=-1)]) == _lib.ERR_INVALID_ARG
    assert wgrad([layer(ck=dict(rows=-1))]) == _lib.ERR_INVALID_ARG
    assert wgrad([layer(ck=dict(q=None))]) == _lib.ERR_INVALID_ARG
    assert wgrad([layer(ck=dict(e=FAKE + 8))]) == _lib.ERR_ALIGNMENT
    assert wgrad([layer(dy=None)]) == _lib.ERR_INVALID_ARG
    assert wgrad([layer(dy=FAKE + 2)]) == _lib.ERR_ALIGNMENT
    assert wgrad([layer(grad=None)]) == _lib.ERR_INVALID_ARG
    assert wgrad([layer(grad=FAKE + 4)]) == _lib.ERR_ALIGNMENT
    assert wgrad([layer(ld_dy=23)]) == _lib.ERR_INVALID_ARG
    assert wgrad([layer(ld_dy=1 << 60)]) == _lib.ERR_UNSUPPORTED
    assert wgrad([layer(rows=(1 << 24) + 1)]) == _lib.ERR_UNSUPPORTED
    assert wgrad([layer(ck=dict(rows=1 << 31))]) == _lib.ERR_UNSUPPORTED
    assert wgrad([layer()], dt=9) == _lib.ERR_INVALID_ARG
    assert wgrad([layer()], dtg=9) == _lib.ERR_INVALID_ARG
    assert wgrad([layer()], acc=-1) == _lib.ERR_INVALID_ARG
    assert wgrad([layer()], ws=None) == _lib.ERR_WORKSPACE
    assert wgrad([layer()], ws=WS + 16) == _lib.ERR_ALIGNMENT
    need = L.iso_workspace_size_weight_grad(iso._weight_grads([layer()]), 1, iso.BF16)
    assert need >= 256 and wgrad([layer()], ws_bytes=need - 1) == _lib.ERR_WORKSPACE
    assert L.iso_workspace_size_weight_grad(iso._weight_grads([layer(rows=-1)]), 1, iso.BF16) == 0
    assert L.iso_workspace_size_weight_grad(None, 1, iso.BF16) == 0
    assert L.iso_ckpt_weight_grad(None, 1, iso.BF16, iso.F32, 0, WS, 1 << 30, None) == _lib.ERR_INVALID_ARG
    with pytest.raises(ValueError):
        iso.weight_grad_workspace([layer(rows=-1)], iso.BF16, "cpu")


def test_status_string_of_a_bad_id():
    assert iso.iso_status_string(_lib.ERR_INDEX) == "token id outside the vocabulary"
