"""What the layer norm and the calls on rows of logits refuse on the host (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2010_08899_b200 import binding as B

INV, WS, UNS = B.DCT_ERR_INVALID_ARG, B.DCT_ERR_WORKSPACE, B.DCT_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def p():
    buf = (ctypes.c_char * (1 << 16))()
    p.keep = buf
    return (ctypes.addressof(buf) + 255) & ~255


def _with(base, **change):
    names = list(base)
    assert all(k in names for k in change)
    return [change.get(k, base[k]) for k in names]


def test_layer_norm_forward_refusals(p):
    ok = dict(x=p, dtype=0, rows=2, d=8, ld=8, w=p + 4096, b=p + 8192, pd=0, eps=1e-5, y=p + 16384, ld_y=8, mean=None, rstd=None,
              stream=None)
    call = lambda **c: B.lib().dct_layer_norm_fwd(*_with(ok, **c))
    for change in (dict(x=None), dict(y=None), dict(d=0), dict(d=65537, ld=65537, ld_y=65537), dict(ld=7), dict(ld_y=7),
                   dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(x=p + 2), dict(y=p + 16385),
                   dict(w=p + 4097), dict(b=p + 8194), dict(mean=p + 2), dict(rstd=p + 1), dict(y=p + 4), dict(y=p, ld_y=9),
                   dict(w=p + 16384), dict(b=p + 16380 + 32)):
        assert call(**change) == INV, change
    for change in (dict(dtype=2), dict(pd=7)):
        assert call(**change) == UNS, change
    assert call(rows=0, x=None, y=None) == B.DCT_OK


def test_layer_norm_backward_refusals(p):
    ok = dict(dy=p, ld_dy=8, x=p + 1024, dtype=0, rows=2, d=8, ld=8, w=p + 2048, pd=0, mean=p + 3328, rstd=p + 3584, dx=p + 4096,
              ld_dx=8, dw=p + 5120, db=p + 6144, ws=p + 8192, nbytes=1 << 15, stream=None)
    call = lambda **c: B.lib().dct_layer_norm_bwd(*_with(ok, **c))
    for change in (dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(dx=None), dict(d=0), dict(ld=7),
                   dict(ld_dy=7), dict(ld_dx=7), dict(dy=p + 2), dict(dx=p + 4097), dict(dw=p + 5121), dict(db=p + 6146),
                   dict(dx=p + 4), dict(dx=p + 1024 + 8), dict(w=p + 4096), dict(dx=p, ld_dx=9)):
        assert call(**change) == INV, change
    for change in (dict(dtype=3), dict(pd=2)):
        assert call(**change) == UNS, change
    need = B.dct_layer_norm_bwd_workspace_bytes(2, 8)
    for change in (dict(ws=None), dict(ws=p + 8192 + 8), dict(nbytes=need - 1)):
        assert call(**change) == WS, change
    assert B.dct_layer_norm_bwd_workspace_bytes(2, 0) == 0 and B.dct_layer_norm_bwd_workspace_bytes(2, 65537) == 0
    assert B.dct_layer_norm_bwd_workspace_bytes((1 << 32) - 1, 65536) < 1 << 30
    assert need % 256 == 0 and need > 0


def test_logprobs_forward_refusals(p):
    ok = dict(x=p, dtype=0, rows=2, vocab=8, ld=8, inv_t=1.0, tok=p + 1024, top=2, lp=p + 2048, ent=p + 3328, st=p + 4096,
              ids=p + 5120, tlp=p + 6144, res=None, stream=None)
    call = lambda **c: B.lib().dct_lm_logprobs_fwd(*_with(ok, **c))
    for change in (dict(x=None), dict(vocab=0), dict(vocab=(1 << 20) + 1, ld=(1 << 20) + 1), dict(ld=7), dict(inv_t=0.0),
                   dict(inv_t=-1.0), dict(inv_t=float("nan")), dict(inv_t=float("inf")), dict(tok=None), dict(lp=None),
                   dict(top=9), dict(vocab=1000, ld=1000, top=257), dict(ids=None), dict(tlp=None), dict(x=p + 2),
                   dict(tok=p + 1025), dict(lp=p + 2050), dict(ent=p + 3073), dict(st=p + 4098), dict(ids=p + 5121),
                   dict(tlp=p + 6146), dict(res=p + 4)):
        assert call(**change) == INV, change
    assert call(dtype=2) == UNS
    assert call(rows=0, x=None) == B.DCT_OK


def test_logprobs_backward_refusals(p):
    ok = dict(x=p, dtype=1, rows=2, vocab=8, ld=8, inv_t=1.0, tok=p + 1024, st=p + 2048, ent=p + 3328, glp=p + 4096, gent=p + 5120,
              g=p + 6144, ld_g=8, stream=None)
    call = lambda **c: B.lib().dct_lm_logprobs_bwd(*_with(ok, **c))
    for change in (dict(x=None), dict(st=None), dict(g=None), dict(tok=None), dict(ent=None), dict(vocab=0), dict(ld=7),
                   dict(ld_g=7), dict(inv_t=0.0), dict(x=p + 1), dict(g=p + 6145), dict(tok=p + 1026), dict(st=p + 2049),
                   dict(ent=p + 3073), dict(glp=p + 4098), dict(gent=p + 5121), dict(g=p + 2), dict(g=p, ld_g=9)):
        assert call(**change) == INV, change
    assert call(dtype=9) == UNS
    assert call(rows=0, x=None, st=None, g=None) == B.DCT_OK


def test_distill_refusals(p):
    ok = dict(x=p, dtype=0, rows=2, vocab=8, ld=8, inv_t=1.0, ids=p + 1024, t=p + 2048, top=2, mode=0, gl=p + 3328, loss=p + 4096,
              g=p + 5120, ld_g=8, res=None, stream=None)
    call = lambda **c: B.lib().dct_lm_distill(*_with(ok, **c))
    for change in (dict(x=None), dict(ids=None), dict(t=None), dict(loss=None, g=None), dict(top=0), dict(top=1025), dict(vocab=0),
                   dict(ld=7), dict(ld_g=7), dict(inv_t=0.0), dict(inv_t=float("inf")), dict(x=p + 2), dict(ids=p + 1025),
                   dict(t=p + 2050), dict(gl=p + 3073), dict(loss=p + 4098), dict(g=p + 5121), dict(g=p + 4),
                   dict(g=p, ld_g=9), dict(res=p + 2)):
        assert call(**change) == INV, change
    for change in (dict(dtype=2), dict(mode=2)):
        assert call(**change) == UNS, change
    assert call(rows=0, x=None, ids=None, t=None) == B.DCT_OK


def test_binding_refuses_wrong_buffers():
    f, i, h = torch.zeros(64), torch.zeros(64, dtype=torch.int32), torch.zeros(64, dtype=torch.float16)
    with pytest.raises(ValueError):
        B.dct_layer_norm_fwd(f, 2, 8, 8, None, None, 1e-5, f, 8)                        # host tensors
    with pytest.raises(TypeError):
        B.dct_layer_norm_fwd(h, 2, 8, 8, None, None, 1e-5, h, 8)
    with pytest.raises(TypeError):
        B.dct_lm_logprobs_fwd(h, 2, 8, 8, 1.0, i, 0, f)
    with pytest.raises(ValueError):
        B.dct_lm_distill(f, 2, 8, 8, 1.0, i, f, 2, B.DCT_DISTILL_TAIL, None, f)
