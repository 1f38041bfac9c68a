"""Matrices in 8 bits without a GPU: the oracle against torch's e4m3, sizes, and what the library and the binding refuse."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import act8 as o
from paper_2010_08899_b200 import binding as B


def test_oracle_codes_are_those_of_e4m3():
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(o.code_values(), every, equal_nan=True)
    gen = torch.Generator().manual_seed(1)
    x = torch.randn(64, 257, generator=gen) * torch.exp(3 * torch.randn(64, 1, generator=gen))
    x[:, ::7] *= 2.0 ** -12
    x[9, :128], x[10, 5], x[11, 200] = 0.0, float("inf"), float("nan")
    h = o.hold(x.double().numpy())
    e = torch.from_numpy(np.repeat(h.bytes.astype(np.int32) - 127, 128, axis=1)[:, :257].copy())
    want = torch.ldexp(x.double(), -e).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    fine = np.repeat(h.bytes != 255, 128, axis=1)[:, :257]
    assert np.array_equal(h.codes[fine], want[fine]) and (h.codes[~fine] == 0x7F).all()
    assert (h.bytes[9, 0], h.bytes[10, 0], h.bytes[11, 1], h.bytes[11, 0] != 255) == (0, 255, 255, True)
    y = np.where(np.isfinite(x.double().numpy()), x.double().numpy(), 0.0)
    assert (np.abs(o.values(o.hold(y)) - y) <= o.half_step(y)).all()
    # the power is the smallest with which the block fits
    largest = np.abs(np.pad(y, ((0, 0), (0, 384 - 257))).reshape(64, 3, 128)).max(2)
    power = np.ldexp(448.0, o.hold(y).bytes.astype(int) - 127)
    assert (largest <= power).all() and ((largest > power / 2) | (o.hold(y).bytes == 0)).all()


def test_oracle_activations_against_known_values_and_differences():
    """SILU is g sigmoid(g); GELU in its tanh form is torch's; the slopes are differences of the values."""
    g = np.linspace(-9, 9, 721)
    t = torch.from_numpy(g)
    assert np.allclose(o.activation(g, False)[0], torch.nn.functional.silu(t).numpy(), rtol=1e-12, atol=1e-15)
    assert np.allclose(o.activation(g, True)[0], torch.nn.functional.gelu(t, approximate="tanh").numpy(), rtol=1e-9, atol=1e-12)
    for gelu in (False, True):
        # a value of up to 9 from four roundings is off by 4 * 9 * 2^-53 = 4e-15, the difference of two by twice that over 2e-6: 4e-9
        slope = (o.activation(g + 1e-6, gelu)[0] - o.activation(g - 1e-6, gelu)[0]) / 2e-6
        assert np.allclose(o.activation(g, gelu)[1], slope, rtol=0, atol=4e-9)


def test_scale_bytes():
    assert B.dct_act8_scale_bytes(1, 1) == 512 and B.dct_act8_scale_bytes(128, 512) == 512
    assert B.dct_act8_scale_bytes(129, 513) == 4 * 512 and B.dct_act8_scale_bytes(0, 5) == 0 and B.dct_act8_scale_bytes(5, 0) == 0
    assert B.dct_act8_scale_bytes(B.DCT_ACT8_MAX_DIM + 1, 1) == 0
    for rows, cols in ((1, 1), (129, 513), (300, 4097)):
        at = o.scale_index(rows, cols)
        assert np.unique(at).size == at.size and at.max() < B.dct_act8_scale_bytes(rows, cols)


# ---- refusals: the addresses are made up, nothing of them is touched ----

def mat(n, rows, cols, ld=None, codes=None, scales=None):
    """The n-th made-up matrix."""
    base = (n + 1) * (1 << 32)
    return B._Act8(base if codes is None else codes, base + (1 << 31) if scales is None else scales, rows, cols,
                   (cols + 15) // 16 * 16 if ld is None else ld, 0)


def at(m):
    return None if m is None else ctypes.addressof(m)


BAD, UNSUPPORTED = B.DCT_ERR_INVALID_ARG, B.DCT_ERR_UNSUPPORTED


@pytest.mark.parametrize("broken", [
    dict(ld=200), dict(ld=112), dict(codes=(1 << 32) + 8), dict(scales=(1 << 32) + 4), dict(codes=0), dict(scales=0),
    dict(rows=9), dict(cols=119)])
def test_unusable_descriptors_are_refused_everywhere(broken):
    L = B.lib()
    size = {k: broken.pop(k) for k in ("rows", "cols") if k in broken}
    def one(n, rows, cols):
        return mat(n, size.get("rows", rows), size.get("cols", cols), **broken)
    x = 90 << 32
    good = [mat(n, 10, 120) for n in range(8)]
    bad = one(20, 10, 120)
    turned = mat(9, 120, 10)
    assert L.dct_act8_pack(x, 0, 10, 120, 120, at(bad), None, None) == BAD
    assert L.dct_act8_pack(x, 0, 10, 120, 120, at(good[0]), at(bad), None) == BAD
    assert L.dct_act8_transpose(at(good[0]), at(bad), None) == BAD
    if not size:
        assert L.dct_act8_unpack(at(bad), x, 0, 120, None) == BAD
        assert L.dct_act8_transpose(at(bad), at(turned), None) == BAD
        assert L.dct_gemm8(at(bad), at(good[0]), None, None, x, 0, 16, 0, None) == BAD
    if "rows" not in size:
        assert L.dct_gemm8(at(good[0]), at(bad), None, None, x, 0, 16, 0, None) == BAD
    assert L.dct_gemm8(at(good[0]), at(good[1]), at(bad), at(good[2]), x, 0, 16, 0, None) == BAD
    assert L.dct_gated8_bwd(x, 0, 120, at(good[0]), at(bad), 0, at(good[2]), None, None, None, None, None) == BAD
    for k in range(5):
        outs = [None] * 5
        outs[k] = at(bad)
        assert L.dct_gated8_bwd(x, 0, 120, at(good[0]), at(good[1]), 0, *outs, None) == BAD
    act, w = mat(30, 10, 64), [mat(31, 120, 64), mat(32, 120, 64)]
    assert L.dct_gated8_fwd(at(act), at(w[0]), at(w[1]), 0, at(bad), None, 0, 0, None, None, None) == BAD
    assert L.dct_gated8_fwd(at(act), at(w[0]), at(w[1]), 0, at(good[0]), None, 0, 0, at(good[1]), at(bad), None) == BAD
    assert L.dct_gated8_fwd(at(act), at(w[0]), at(bad), 0, at(good[0]), None, 0, 0, None, None, None) == BAD


def test_other_refusals():
    L = B.lib()
    x = 90 << 32
    a, b, t = mat(0, 10, 120), mat(1, 40, 120), mat(2, 120, 10)
    # no output, unknown types, short strides, misaligned or missing buffers
    assert L.dct_act8_pack(x, 0, 10, 120, 120, None, None, None) == BAD
    assert L.dct_act8_pack(x, 7, 10, 120, 120, at(a), None, None) == UNSUPPORTED
    assert L.dct_act8_pack(x, 0, 10, 120, 119, at(a), None, None) == BAD
    assert L.dct_act8_pack(x + 2, 0, 10, 120, 120, at(a), None, None) == BAD
    assert L.dct_act8_pack(None, 0, 10, 120, 120, at(a), None, None) == BAD
    assert L.dct_act8_unpack(None, x, 0, 120, None) == BAD
    assert L.dct_act8_unpack(at(a), x, 0, 119, None) == BAD
    assert L.dct_act8_unpack(at(a), x + 1, 1, 120, None) == BAD
    assert L.dct_gemm8(at(a), at(b), None, None, x, 9, 40, 0, None) == UNSUPPORTED
    assert L.dct_gemm8(at(a), at(b), None, None, x, 0, 39, 0, None) == BAD
    assert L.dct_gemm8(at(a), at(b), None, None, None, 0, 40, 0, None) == BAD
    assert L.dct_gemm8(at(a), at(t), None, None, x, 0, 120, 0, None) == BAD                   # depths differ
    assert L.dct_gemm8(at(a), at(b), at(a), None, x, 0, 40, 0, None) == BAD
    assert L.dct_gemm8(at(a), at(b), at(b), at(b), x, 0, 40, 0, None) == BAD
    w = [mat(3, 64, 120), mat(4, 64, 120)]
    h, g, u = mat(5, 10, 64), mat(6, 10, 64), mat(7, 10, 64)
    fwd = lambda act=0, h=h, dense=None, dt=0, ld=64, g=None, u=None: L.dct_gated8_fwd(at(a), at(w[0]), at(w[1]), act, at(h), dense, dt,
                                                                                         ld, at(g), at(u), None)
    assert fwd(act=2) == UNSUPPORTED and fwd(dt=3) == UNSUPPORTED and fwd(h=None) == BAD and fwd(g=g) == BAD and fwd(u=u) == BAD
    assert fwd(dense=x, ld=63) == BAD and fwd(dense=x + 1, dt=1) == BAD
    dg = mat(8, 10, 64)
    bwd = lambda dh=x, dt=0, ld=64, act=0, out=dg: L.dct_gated8_bwd(dh, dt, ld, at(g), at(u), act, at(out), None, None, None, None, None)
    assert bwd(out=None) == BAD and bwd(dt=5) == UNSUPPORTED and bwd(act=-1) == UNSUPPORTED and bwd(ld=63) == BAD and bwd(dh=None) == BAD
    assert bwd(dh=x + 2) == BAD


def test_outputs_may_overlap_nothing():
    L = B.lib()
    x = 90 << 32
    a, b, t = mat(0, 10, 120), mat(1, 40, 120), mat(2, 120, 10)
    assert L.dct_act8_pack(a.codes + 64, 0, 10, 120, 120, at(a), None, None) == BAD
    assert L.dct_act8_pack(a.scales, 0, 10, 120, 120, at(a), None, None) == BAD
    assert L.dct_act8_pack(x, 0, 10, 120, 120, at(a), at(mat(2, 120, 10, codes=a.codes)), None) == BAD
    assert L.dct_act8_pack(x, 0, 10, 120, 120, at(a), at(mat(2, 120, 10, scales=a.scales)), None) == BAD
    assert L.dct_act8_unpack(at(a), a.codes, 0, 120, None) == BAD
    assert L.dct_act8_transpose(at(a), at(mat(2, 120, 10, codes=a.codes + 16)), None) == BAD
    assert L.dct_gemm8(at(a), at(b), None, None, a.codes, 0, 40, 0, None) == BAD
    assert L.dct_gemm8(at(a), at(b), None, None, b.scales, 0, 40, 0, None) == BAD
    h, g, u = mat(5, 10, 64), mat(6, 10, 64), mat(7, 10, 64)
    w = [mat(3, 64, 120), mat(4, 64, 120)]
    assert L.dct_gated8_fwd(at(a), at(w[0]), at(w[1]), 0, at(h), None, 0, 0, at(h), at(u), None) == BAD
    assert L.dct_gated8_fwd(at(a), at(w[0]), at(w[1]), 0, at(h), h.codes, 0, 64, None, None, None) == BAD
    assert L.dct_gated8_bwd(x, 0, 64, at(g), at(u), 0, at(g), None, None, None, None, None) == BAD
    assert L.dct_gated8_bwd(h.codes, 0, 64, at(g), at(u), 0, at(h), None, None, None, None, None) == BAD
    # columns of one wider buffer that share a few
    wide = 1 << 40
    left, bad = mat(0, 10, 64, ld=128, codes=wide), mat(1, 10, 64, ld=128, codes=wide + 48)
    assert L.dct_gated8_bwd(x, 0, 64, at(g), at(u), 0, at(left), at(bad), None, None, None, None) == BAD


def test_empty_matrices_need_no_buffers():
    """Nothing is launched (this runs without a GPU)."""
    L = B.lib()
    none = B._Act8(None, None, 0, 120, 0, 0)
    turned = B._Act8(None, None, 120, 0, 0, 0)
    w, u = mat(3, 64, 120), mat(4, 64, 120)
    h = B._Act8(None, None, 0, 64, 0, 0)
    assert L.dct_act8_pack(None, 0, 0, 120, 120, at(none), at(turned), None) == B.DCT_OK
    assert L.dct_act8_unpack(at(none), None, 0, 120, None) == B.DCT_OK
    assert L.dct_act8_transpose(at(none), at(turned), None) == B.DCT_OK
    assert L.dct_gemm8(at(none), at(w), None, None, None, 0, 64, 0, None) == B.DCT_OK
    assert L.dct_gated8_fwd(at(none), at(w), at(u), 0, at(h), None, 0, 0, at(h), at(h), None) == B.DCT_OK
    assert L.dct_gated8_bwd(None, 0, 64, at(h), at(h), 0, at(h), None, None, None, None, None) == B.DCT_OK


def test_the_binding_refuses_what_is_no_matrix():
    host = torch.zeros(4, 32, dtype=torch.uint8)
    with pytest.raises(ValueError):
        B.act8(host, host, 4, 32)                                   # not on a GPU
    with pytest.raises(TypeError):
        B.act8(host.float(), host, 4, 32)
    for rows, cols in ((-1, 8), (8, -1), (1 << 29, 8)):
        with pytest.raises(ValueError):
            B.act8(host, host, rows, cols)
