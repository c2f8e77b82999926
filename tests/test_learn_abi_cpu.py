"""Refusals of the attention and distillation entry points: every bad argument is answered on the host before anything is
queued.  No GPU is used: the pointers below are never dereferenced."""
import ctypes

import pytest

import paper_2607_19331_amd as iso
from paper_2607_19331_amd import _lib

FAKE = 0x100000
WS = FAKE * 16


def attn(**kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, start_q=FAKE, start_k=FAKE, sequences=2, tokens_q=64, tokens_k=64, heads=4, heads_kv=2,
             dim=64, scale=0.125, out=FAKE, lse=FAKE, dout=FAKE, dq=FAKE, dk=FAKE, dv=FAKE)
    a.update(kw)
    return iso.Attn(**a)


def forward(a, dt=iso.BF16, ws=WS, ws_bytes=1 << 40):
    return _lib.load().iso_attend(ctypes.byref(iso._attn(a)), dt, ws, ws_bytes, None)


def backward(a, dt=iso.BF16, ws=WS, ws_bytes=1 << 40):
    return _lib.load().iso_attend_grad(ctypes.byref(iso._attn(a)), dt, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [forward, backward])
def test_attend_refusals(call):
    for kw in (dict(sequences=-1), dict(tokens_q=-1), dict(tokens_k=-1), dict(heads=0), dict(heads_kv=0), dict(heads=5), dict(dim=0),
               dict(window=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
               dict(scale=1e300), dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(lse=None), dict(start_q=None),
               dict(start_k=None), dict(ld_q=248), dict(ld_k=120), dict(ld_v=0), dict(ld_out=8), dict(heads=-4, heads_kv=-2)):
        assert call(attn(**kw)) == _lib.ERR_INVALID_ARG, kw
    a = iso._attn(attn())
    a.causal = 2
    assert _lib.load().iso_attend(ctypes.byref(a), iso.BF16, WS, 1 << 40, None) == _lib.ERR_INVALID_ARG
    assert call(attn(), dt=2) == _lib.ERR_INVALID_ARG
    for kw in (dict(q=FAKE + 8), dict(k=FAKE + 2), dict(v=FAKE + 4), dict(out=FAKE + 8), dict(lse=FAKE + 4), dict(start_q=FAKE + 2),
               dict(start_k=FAKE + 1), dict(ld_q=260), dict(ld_k=129), dict(ld_v=132), dict(ld_out=257)):
        assert call(attn(**kw)) == _lib.ERR_ALIGNMENT, kw
    for kw in (dict(dim=60), dict(dim=136), dict(sequences=_lib.ATTN_MAX_SEQUENCES + 1), dict(ld_q=_lib.ATTN_MAX_LD + 8),
               dict(heads=1 << 16, heads_kv=1), dict(heads=1025, heads_kv=1, dim=8), dict(tokens_q=(_lib.ATTN_MAX_ROWS >> 2) + 1),
               dict(tokens_k=(_lib.ATTN_MAX_ROWS >> 1) + 1), dict(heads=512, heads_kv=512, dim=8, sequences=(1 << 13) + 1),
               dict(tokens_q=1 << 40), dict(tokens_k=1 << 31), dict(tokens_q=(1 << 63) - 1)):
        assert call(attn(**kw)) == _lib.ERR_UNSUPPORTED, kw
    assert call(attn(), ws=None) == _lib.ERR_WORKSPACE
    assert call(attn(), ws_bytes=255) == _lib.ERR_WORKSPACE
    assert call(attn(), ws=WS + 128) == _lib.ERR_ALIGNMENT
    # a stride of four floats is whole 16 bytes; the workspace is checked last
    assert call(attn(ld_q=260, ld_out=260), dt=iso.F32, ws_bytes=0) == _lib.ERR_WORKSPACE


def test_attend_grad_refusals():
    for kw in (dict(dout=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(ld_dout=9), dict(ld_dq=0), dict(ld_dk=1),
               dict(ld_dv=127)):
        assert backward(attn(**kw)) == _lib.ERR_INVALID_ARG, kw
    for kw in (dict(dout=FAKE + 8), dict(dq=FAKE + 2), dict(dk=FAKE + 4), dict(dv=FAKE + 8), dict(ld_dout=257), dict(ld_dq=258),
               dict(ld_dk=130), dict(ld_dv=132)):
        assert backward(attn(**kw)) == _lib.ERR_ALIGNMENT, kw
    L = _lib.load()
    assert L.iso_attend(None, iso.BF16, WS, 1 << 40, None) == _lib.ERR_INVALID_ARG
    assert L.iso_attend_grad(None, iso.BF16, WS, 1 << 40, None) == _lib.ERR_INVALID_ARG
    assert L.iso_workspace_size_attend(None, iso.BF16, 0) == 0
    assert L.iso_workspace_size_attend(ctypes.byref(iso._attn(attn(dim=12))), iso.BF16, 0) == 0
    assert L.iso_workspace_size_attend(ctypes.byref(iso._attn(attn())), iso.BF16, 2) == 0
    assert L.iso_workspace_size_attend(ctypes.byref(iso._attn(attn())), 7, 1) == 0
    with pytest.raises(ValueError):
        iso.attend_workspace(attn(heads=3), iso.BF16, device="cpu")
    with pytest.raises(iso.IsoError, match="invalid argument"):
        iso.iso_attend(attn(q=None), iso.BF16, stream=0)
    with pytest.raises(iso.IsoError, match="invalid argument"):
        iso.iso_attend_grad(attn(dq=None), iso.BF16, stream=0)


@pytest.mark.parametrize("dt", [iso.F32, iso.BF16])
@pytest.mark.parametrize("grad", [0, 1])
def test_attend_workspaces_hold_smaller_calls(dt, grad):
    need = lambda **kw: _lib.load().iso_workspace_size_attend(ctypes.byref(iso._attn(attn(**kw))), dt, grad)  # noqa: E731
    call = backward if grad else forward
    for kw in (dict(heads=28, heads_kv=4, dim=128), dict(heads=3, heads_kv=3, dim=8), dict(heads=64, heads_kv=1, dim=72)):
        last = 0
        for sequences, q, k in ((0, 0, 0), (1, 1, 1), (1, 1, 9), (1, 1, 4000), (1, 1, 20000), (3, 9, 20000), (3, 100, 20000),
                                (3, 1000, 20000), (7, 5000, 20000), (7, 20000, 20000), (90, 20000, 30000), (90, 90000, 90000)):
            n = need(sequences=sequences, tokens_q=q, tokens_k=k, **kw)
            assert n >= max(last, 256) and n % 256 == 0
            assert call(attn(sequences=sequences, tokens_q=q, tokens_k=k, **kw), dt=dt, ws_bytes=n - 1) == _lib.ERR_WORKSPACE
            last = n


def distill(**kw):
    a = dict(logits=FAKE, tokens=4, vocab=100, ids=FAKE, teacher=FAKE, top=5, loss=FAKE, lse=FAKE, grad=FAKE * 2, weight=FAKE,
             id_type=_lib.I64)
    a.update(kw)
    return iso.Distill(**a)


def loss(d, dt=iso.BF16, ws=WS, ws_bytes=1 << 30):
    return _lib.load().iso_distill_loss(ctypes.byref(iso._distill(d)), dt, ws, ws_bytes, None)


def gradient(d, dt=iso.BF16, ws=WS, ws_bytes=1 << 30):
    return _lib.load().iso_distill_grad(ctypes.byref(iso._distill(d)), dt, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [loss, gradient])
def test_distill_refusals(call):
    for kw in (dict(tokens=-1), dict(vocab=0), dict(top=0), dict(id_type=2), dict(ids=None), dict(logits=None), dict(teacher=None),
               dict(lse=None), dict(ld=99), dict(ld_grad=99), dict(temperature=0.0), dict(temperature=-1.0),
               dict(temperature=float("nan")), dict(temperature=float("inf")), dict(temperature=1e-300), dict(temperature=4e-39),
               dict(temperature=1e300),
               dict(grad=FAKE, ld_grad=104)):
        assert call(distill(**kw)) == _lib.ERR_INVALID_ARG, kw
    assert call(distill(), dt=3) == _lib.ERR_INVALID_ARG
    for kw in (dict(logits=FAKE + 8), dict(ids=FAKE + 4), dict(teacher=FAKE + 4), dict(lse=FAKE + 8), dict(weight=FAKE + 2),
               dict(grad=FAKE + 2)):
        assert call(distill(**kw)) == _lib.ERR_ALIGNMENT, kw
    for kw in (dict(tokens=1 << 31), dict(tokens=_lib.DISTILL_MAX_TOKENS + 1), dict(vocab=_lib.EMBED_MAX_VOCAB + 1), dict(top=_lib.DISTILL_MAX_TOP + 1), dict(ld=1 << 60),
               dict(ld_grad=1 << 60)):
        assert call(distill(**kw)) == _lib.ERR_UNSUPPORTED, kw
    assert call(distill(), ws=None) == _lib.ERR_WORKSPACE
    assert call(distill(), ws=WS + 8) == _lib.ERR_ALIGNMENT
    need = _lib.load().iso_workspace_size_distill(ctypes.byref(iso._distill(distill())))
    assert need >= 256 and call(distill(), ws_bytes=need - 1) == _lib.ERR_WORKSPACE
    assert call(distill(ids=FAKE + 4, id_type=_lib.I32), ws_bytes=0) == _lib.ERR_WORKSPACE


def test_more_distill_refusals():
    L = _lib.load()
    assert loss(distill(loss=None)) == _lib.ERR_INVALID_ARG
    assert loss(distill(loss=FAKE + 8)) == _lib.ERR_ALIGNMENT
    assert gradient(distill(grad=None)) == _lib.ERR_INVALID_ARG
    assert loss(distill(grad=None, ld_grad=0), ws_bytes=0) == _lib.ERR_WORKSPACE          # a loss alone
    assert gradient(distill(loss=None), ws_bytes=0) == _lib.ERR_WORKSPACE                 # a gradient alone
    assert L.iso_distill_loss(None, iso.BF16, WS, 1 << 30, None) == _lib.ERR_INVALID_ARG
    assert L.iso_distill_grad(None, iso.BF16, WS, 1 << 30, None) == _lib.ERR_INVALID_ARG
    assert L.iso_workspace_size_distill(None) == 0
    size = lambda **kw: L.iso_workspace_size_distill(ctypes.byref(iso._distill(distill(**kw))))  # noqa: E731
    assert size(top=0) == 0 and size(tokens=1) <= size(tokens=100) <= size(tokens=100000)
    with pytest.raises(ValueError):
        iso.distill_workspace(distill(vocab=0), "cpu")
    with pytest.raises(TypeError):
        iso._distill(distill(id_type=None))
    with pytest.raises(iso.IsoError, match="invalid argument"):
        iso.iso_distill_loss(distill(ids=None), iso.BF16, stream=0)
    with pytest.raises(iso.IsoError, match="invalid argument"):
        iso.iso_distill_grad(distill(lse=None), iso.BF16, stream=0)
