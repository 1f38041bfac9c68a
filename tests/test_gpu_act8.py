"""Matrices in 8 bits on the GPU against the 64-bit oracle: what is written is the oracle's to the bit; products and the gated block are
within what fp32 sums and one rounding allow."""
import numpy as np
import pytest
import torch

from oracle import act8 as o
from paper_2010_08899_b200 import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPES = [torch.float32, torch.bfloat16]
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}      # half a step, relative


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def rows_of(rows, cols, dtype=torch.float32, seed=0, pad=0, offset=0):
    """[rows, cols + pad] of ``dtype``, `offset` elements past a boundary, rows of different size; the columns behind hold what no
    result may show."""
    g = gen(seed)
    x = torch.randn(rows, cols + pad, generator=g, device=DEV) * torch.exp(torch.randn(rows, 1, generator=g, device=DEV))
    x[:, cols:] = float("nan")
    buf = torch.empty(x.numel() + offset + 64, dtype=dtype, device=DEV)
    base = (-buf.data_ptr() % 256) // buf.element_size()
    view = buf[base + offset: base + offset + x.numel()].view(rows, cols + pad)
    view.copy_(x)
    return view


class Guarded:
    """A matrix in 8 bits whose buffers are longer and wider than it needs, filled with marks."""

    def __init__(self, rows, cols, wider=16):
        ld = (cols + 15) // 16 * 16 + wider
        self.codes = torch.full((rows + 2, ld), 0xAB, dtype=torch.uint8, device=DEV)
        need = B.dct_act8_scale_bytes(rows, cols)
        self.scales = torch.full((need + 64,), 0xCD, dtype=torch.uint8, device=DEV)
        self.a = B.act8(self.codes[1:], self.scales, rows, cols)
        self.rows, self.cols, self.need = rows, cols, need

    def read(self):
        """The oracle's form of what was written, after a look at the marks."""
        c, s = self.codes.cpu().numpy(), self.scales.cpu().numpy()
        assert (c[0] == 0xAB).all() and (c[-1] == 0xAB).all() and (c[:, self.cols:] == 0xAB).all(), "codes outside the matrix"
        assert (s[self.need:] == 0xCD).all(), "scales outside the matrix"
        return o.Held(c[1:-1, :self.cols], s[o.scale_index(self.rows, self.cols)])


def put(h: o.Held, wider=16):
    """A matrix in 8 bits from the oracle's form; what does not count holds marks (NaN codes and powers among them)."""
    g = Guarded(*h.codes.shape, wider=wider)
    g.codes[1:-1, :g.cols] = torch.from_numpy(h.codes).to(DEV)
    g.codes[1:-1, g.cols:] = 0x7F
    s = np.full(g.scales.numel(), 255, np.uint8)
    s[o.scale_index(g.rows, g.cols)] = h.bytes
    g.scales.copy_(torch.from_numpy(s))
    return g.a


def f64(t):
    return t.detach().double().cpu().numpy()


def same(got: o.Held, want: o.Held):
    assert np.array_equal(got.bytes, want.bytes)
    assert np.array_equal(got.codes, want.codes)


SHAPES = [(1, 1, 0, 0), (1, 128, 0, 0), (3, 129, 0, 0), (8, 4096, 0, 0), (127, 8, 8, 0), (128, 128, 0, 0), (129, 257, 3, 1),
          (200, 1000, 5, 1), (261, 640, 0, 3), (385, 77, 0, 0), (1000, 15, 1, 0), (5, 5003, 0, 7)]


# ---- writing, reading, transposing ----

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad,offset", SHAPES)
def test_pack(rows, cols, pad, offset, dtype):
    x = rows_of(rows, cols, dtype, rows + cols, pad, offset)
    ld = cols + pad
    v = f64(x)[:, :cols]
    for by_rows, turned in ((True, True), (True, False), (False, True)):
        a, t = Guarded(rows, cols), Guarded(cols, rows, wider=0)
        B.dct_act8_pack(x, rows, cols, ld, a.a if by_rows else None, t.a if turned else None)
        if by_rows:
            same(a.read(), o.hold(v))
        if turned:
            same(t.read(), o.hold(v.T))


@pytest.mark.parametrize("dtype", TYPES)
def test_pack_of_values_at_the_borders(dtype):
    """Zeros, both signs of them, the largest and the smallest numbers, halfway cases, blocks whose largest is 448 2^e or next to it,
    infinities and NaN (their blocks alone are lost)."""
    rows, cols = 40, 384
    x = rows_of(rows, cols, torch.float32, 5)
    x[1], x[2] = 0.0, -0.0
    x[3] = torch.linspace(-450, 450, cols, device=DEV)
    x[4] = torch.arange(cols, device=DEV) * 2.0 ** -10           # every second one halfway, subnormal codes
    x[4, ::128] = 300.0
    x[5], x[5, 0] = 0.0, 448.0
    x[6], x[6, 0] = 1.0, float(np.nextafter(np.float32(448.0), np.float32(1e9)))
    x[7] = torch.finfo(dtype).max
    x[7, 1:] = x[7, 1:] * 2.0 ** -3
    x[8] = 2.0 ** -126
    x[9] = 2.0 ** -133
    x[10, 130], x[11, 200], x[12, 5] = float("inf"), float("-inf"), float("nan")
    x[13] = torch.finfo(dtype).tiny
    x = x.to(dtype)
    a, t = Guarded(rows, cols), Guarded(cols, rows)
    B.dct_act8_pack(x, rows, cols, cols, a.a, t.a)
    v = f64(x)
    same(a.read(), o.hold(v))
    same(t.read(), o.hold(v.T))
    y = torch.empty(rows, cols, device=DEV)
    B.dct_act8_unpack(a.a, y, cols)
    assert torch.isnan(y[10]).sum() == torch.isnan(y[11]).sum() == torch.isnan(y[12]).sum() == 128 and torch.isfinite(y[13:]).all()
    assert (f64(y)[1:3] == 0).all() and y[5, 0] == 448 and np.isfinite(f64(y)[:10]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad,offset", SHAPES)
def test_unpack(rows, cols, pad, offset, dtype):
    h = o.hold(f64(rows_of(rows, cols, seed=rows * 3 + cols)))
    a = put(h)
    buf = torch.full((rows * (cols + pad) + offset + 8,), -3.0, dtype=dtype, device=DEV)
    y = buf[offset:offset + rows * (cols + pad)].view(rows, cols + pad)
    B.dct_act8_unpack(a, y, cols + pad)
    assert np.array_equal(f64(y)[:, :cols], o.values(h))
    assert bool((y[:, cols:] == -3.0).all()) and bool((buf[:offset] == -3.0).all()) and bool((buf[-8:] == -3.0).all())


@pytest.mark.parametrize("rows,cols", [s[:2] for s in SHAPES])
def test_transpose(rows, cols):
    h = o.hold(f64(rows_of(rows, cols, seed=rows * 5 + cols)))
    t = Guarded(cols, rows)
    B.dct_act8_transpose(put(h), t.a)
    same(t.read(), o.hold(o.values(h).T))


def test_transposing_twice_gives_the_same_values():
    """Rows of one size: no value is 2^13 below its new block's largest unless it was far below its old one's."""
    x = torch.randn(300, 520, generator=gen(3), device=DEV)
    x = x.sign() * x.abs().clamp_min(2.0 ** -7)
    a, t, b = B.new_act8(300, 520), B.new_act8(520, 300), B.new_act8(300, 520)
    B.dct_act8_pack(x, 300, 520, 520, a)
    B.dct_act8_transpose(a, t)
    B.dct_act8_transpose(t, b)
    y, z = torch.empty_like(x), torch.empty_like(x)
    B.dct_act8_unpack(a, y, 520)
    B.dct_act8_unpack(b, z, 520)
    assert torch.equal(y, z)


def test_matrices_side_by_side_in_wider_rows():
    x = rows_of(70, 200, torch.bfloat16, 9)
    wide = torch.full((70, 480), 0xAB, dtype=torch.uint8, device=DEV)
    sc = [torch.empty(B.dct_act8_scale_bytes(70, 200), dtype=torch.uint8, device=DEV) for _ in range(2)]
    left, right = B.act8(wide[:, :208], sc[0], 70, 200), B.act8(wide[:, 208:416], sc[1], 70, 200)
    B.dct_act8_pack(x, 70, 200, 200, left)
    B.dct_act8_pack(-x, 70, 200, 200, right)
    assert bool((wide[:, 200:208] == 0xAB).all()) and bool((wide[:, 408:] == 0xAB).all())
    want = o.hold(f64(x))
    assert np.array_equal(wide[:, :200].cpu().numpy(), want.codes)
    assert np.array_equal(wide[:, 208:408].cpu().numpy() ^ 128, want.codes)
    with pytest.raises(B.DctError):         # one column more and they would meet
        B.dct_gated8_bwd(x, 200, left, left, B.DCT_ACT_SILU, B.act8(wide[:, 208:], sc[1], 70, 200), B.act8(wide[:, 400:], sc[0], 70, 80))


# ---- products ----

def matrix(rows, cols, seed):
    return o.hold(f64(rows_of(rows, cols, seed=seed)))


def product_bound(a, b, dtype, want, extra=0.0):
    """Sums of n terms in fp32, in whatever order: each of at most n additions is off by at most 2^-23 of what it has reached (a tensor core
    cuts instead of rounding), which is at most the sum of the magnitudes; then one rounding."""
    n = a.shape[1] + 2
    size = np.abs(a) @ np.abs(b).T + extra
    return n * 2.0 ** -23 * size + HALF[dtype] * (np.abs(want) + n * 2.0 ** -23 * size)


PRODUCTS = [(1, 1, 1), (1, 64, 128), (2, 5003, 640), (16, 512, 4096), (31, 129, 513), (32, 1000, 96), (33, 256, 1024), (64, 2048, 200),
            (65, 384, 2000), (128, 128, 128), (129, 257, 385), (200, 700, 1030), (255, 1000, 3), (300, 1, 700), (520, 1300, 260)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(m, n, k, dtype):
    a, b = matrix(m, k, 1), matrix(n, k, 2)
    va, vb = o.values(a), o.values(b)
    want = va @ vb.T
    for pad, offset in ((0, 0), (5, 1)):
        buf = torch.full((m * (n + pad) + offset + 8,), -3.0, dtype=dtype, device=DEV)
        c = buf[offset:offset + m * (n + pad)].view(m, n + pad)
        B.dct_gemm8(put(a), put(b), c, n + pad)
        got = f64(c)[:, :n]
        assert (np.abs(got - want) <= product_bound(va, vb, dtype, want)).all()
        assert bool((c[:, n:] == -3.0).all()) and bool((buf[:offset] == -3.0).all()) and bool((buf[-8:] == -3.0).all())
        # and as a whole: errors of either sign add up to far less than their bound
        assert np.linalg.norm(got - want) <= (1e-5 + HALF[dtype]) * np.linalg.norm(want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(2400, 4200, 900), (300, 40000, 260), (60, 20000, 300), (128, 300, 20000), (4100, 520, 8200)])
def test_product_of_many_tiles_or_great_depth(m, n, k, dtype):
    """More tiles than the device has SMs, and depths that several CTAs share; compared in 64 bits on the device."""
    a, b = matrix(m, k, 1), matrix(n, k, 2)
    va, vb = torch.from_numpy(o.values(a)).to(DEV), torch.from_numpy(o.values(b)).to(DEV)
    want, size = va @ vb.T, va.abs() @ vb.abs().T
    c = torch.empty(m, n, dtype=dtype, device=DEV)
    pa, pb = put(a), put(b)
    B.dct_gemm8(pa, pb, c, n)
    off = (c.double() - want).abs()
    assert bool((off <= (k + 2) * 2.0 ** -23 * size * (1 + HALF[dtype]) + HALF[dtype] * want.abs()).all())
    assert float(off.norm() / want.norm()) <= 1e-5 + HALF[dtype]
    again = torch.empty_like(c)
    B.dct_gemm8(pa, pb, again, n)
    assert torch.equal(c, again)


@pytest.mark.parametrize("m,n,k,k2", [(1, 100, 64, 700), (20, 300, 513, 129), (70, 200, 1, 1), (150, 300, 640, 1100), (260, 520, 1300, 2)])
def test_two_products_added_to_what_is_there(m, n, k, k2):
    a, b, a2, b2 = matrix(m, k, 1), matrix(n, k, 2), matrix(m, k2, 3), matrix(n, k2, 4)
    va, vb = np.concatenate([o.values(a), o.values(a2)], 1), np.concatenate([o.values(b), o.values(b2)], 1)
    for dtype in TYPES:
        c0 = torch.randn(m, n, generator=gen(5), device=DEV).to(dtype)
        for accumulate in (False, True):
            c = c0.clone()
            B.dct_gemm8(put(a), put(b), c, n, put(a2), put(b2), accumulate)
            before = f64(c0) if accumulate else 0.0
            want = va @ vb.T + before
            assert (np.abs(f64(c) - want) <= product_bound(va, vb, dtype, want, np.abs(before))).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k,k2", [(2300, 4300, 4200, 130), (2560, 4352, 100, 9000), (2300, 4300, 1, 1)])
def test_two_products_of_many_tiles(m, n, k, k2, dtype):
    """The same over pairs of CTAs, whose sums into fp32 come in pieces that the second product may begin in; C starts on no boundary."""
    a, b, a2, b2 = matrix(m, k, 1), matrix(n, k, 2), matrix(m, k2, 3), matrix(n, k2, 4)
    on = lambda h: torch.from_numpy(o.values(h)).to(DEV)
    va, vb = torch.cat([on(a), on(a2)], 1), torch.cat([on(b), on(b2)], 1)
    product, size = va @ vb.T, va.abs() @ vb.abs().T
    pa, pb, pa2, pb2 = put(a), put(b), put(a2), put(b2)
    for pad, offset, accumulate in ((0, 0, True), (3, 1, True), (3, 1, False)):
        buf = torch.randn(m * (n + pad) + offset + 8, generator=gen(5), device=DEV).to(dtype)
        before = buf.clone()
        c = buf[offset:offset + m * (n + pad)].view(m, n + pad)
        was = before[offset:offset + m * (n + pad)].view(m, n + pad)[:, :n].double() * accumulate
        B.dct_gemm8(pa, pb, c, n + pad, pa2, pb2, accumulate)
        want, terms = product + was, k + k2 + 3
        off = (c[:, :n].double() - want).abs()
        assert bool((off <= terms * 2.0 ** -23 * (size + was.abs()) * (1 + HALF[dtype]) + HALF[dtype] * want.abs()).all())
        assert torch.equal(c[:, n:], before[offset:offset + m * (n + pad)].view(m, n + pad)[:, n:]) and torch.equal(buf[-8:], before[-8:])


def test_product_without_depth_into_far_rows():
    """Rows of C more than 2 GiB apart."""
    n, ld = 300, (1 << 30) + 24
    a, b = B.new_act8(3, 0), B.new_act8(n, 0)
    c = torch.full((2 * ld + n + 8,), 2.0, dtype=torch.bfloat16, device=DEV)
    B.dct_gemm8(a, b, c, ld)
    for r in range(3):
        assert float(c[r * ld:r * ld + n].abs().max()) == 0.0 and float(c[r * ld + n:r * ld + n + 8].min()) == 2.0


@pytest.mark.parametrize("m,n", [(5, 300), (200, 300)])
def test_product_without_depth(m, n):
    """The gradient of weights from a batch of no rows: zeros, or what was there."""
    empty = lambda r: B.act8(torch.empty(r, 0, dtype=torch.uint8, device=DEV), torch.empty(0, dtype=torch.uint8, device=DEV), r, 0)
    for dtype in TYPES:
        c = torch.full((m, n + 3), 2.0, dtype=dtype, device=DEV)
        B.dct_gemm8(empty(m), empty(n), c, n + 3, accumulate=True)
        assert bool((c == 2.0).all())
        B.dct_gemm8(empty(m), empty(n), c, n + 3)
        assert bool((c[:, :n] == 0.0).all()) and bool((c[:, n:] == 2.0).all())
        a, b = matrix(m, 70, 1), matrix(n, 70, 2)
        d = torch.empty(m, n, dtype=dtype, device=DEV)
        B.dct_gemm8(empty(m), empty(n), d, n, put(a), put(b))
        e = torch.empty(m, n, dtype=dtype, device=DEV)
        B.dct_gemm8(put(a), put(b), e, n)
        assert torch.equal(d, e)


@pytest.mark.parametrize("m,n,k", [(9, 300, 700), (300, 400, 700)])
def test_a_lost_block_is_lost_in_its_row_alone(m, n, k):
    x, y = rows_of(m, k, seed=1), rows_of(n, k, seed=2)
    x[m // 2, k - 1] = float("nan")
    y[n - 1, 0] = float("inf")
    a, b = o.hold(f64(x)), o.hold(f64(y))
    c = torch.empty(m, n, device=DEV)
    B.dct_gemm8(put(a), put(b), c, n)
    lost = torch.isnan(c).cpu().numpy()
    want = np.zeros((m, n), bool)
    want[m // 2], want[:, n - 1] = True, True
    assert np.array_equal(lost, want)


def test_product_of_far_apart_powers():
    """Blocks at the ends of fp32's range: powers multiply without overflow on the way, and what is below fp32 is 0."""
    m, n, k = 130, 256, 512
    x, y = rows_of(m, k, seed=3), rows_of(n, k, seed=4)
    x *= torch.exp2(torch.linspace(-100, 50, m, device=DEV))[:, None]
    y *= torch.exp2(torch.linspace(-40, 60, n, device=DEV))[:, None]
    y[0], x[0] = 0.0, 0.0
    a, b = o.hold(f64(x)), o.hold(f64(y))
    va, vb = o.values(a), o.values(b)
    c = torch.empty(m, n, device=DEV)
    B.dct_gemm8(put(a), put(b), c, n)
    want = va @ vb.T
    assert (np.abs(f64(c) - want) <= product_bound(va, vb, torch.float32, want) + 2.0 ** -126 * k).all()


# ---- the gated block ----

GATED = [(2, 200, 20000), (900, 130, 2500), (1, 128, 64), (3, 700, 130), (16, 512, 1000), (40, 300, 129), (64, 96, 257), (100, 1, 1), (130, 256, 384), (300, 640, 520), (9, 2100, 300)]


def near_held(got: o.Held, want, off):
    """What was rounded from a number within ``off`` of want: half a step of 8 bits, at its own power (next to a border the power may be
    either one; the larger one's step counts)."""
    v = o.values(got)
    return (np.abs(v - want) <= off + np.maximum(o.half_step(want + off), o.half_step(want - off)) + 2.0 ** -12 * np.abs(want)).all()


@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("rows,d,f", GATED)
def test_gated_forward(rows, d, f, gelu):
    x, wg, wu = matrix(rows, d, 1), o.hold(f64(rows_of(f, d, seed=2)) * d ** -0.5), o.hold(f64(rows_of(f, d, seed=3)) * d ** -0.5)
    vx, vg, vu = o.values(x), o.values(wg), o.values(wu)
    g, u = vx @ vg.T, vx @ vu.T
    act, slope = o.activation(g, gelu)
    n = d + 2
    off_g, off_u = n * 2.0 ** -23 * (np.abs(vx) @ np.abs(vg).T), n * 2.0 ** -23 * (np.abs(vx) @ np.abs(vu).T)
    # |act'| is below 1.13; the share itself: its argument's rounding (up to 2^-21 of |y|, and |y| q is below 1), a few steps of exp and the quotient
    off_h = 1.13 * off_g * (np.abs(u) + off_u) + np.abs(act) * off_u + 2.0 ** -18 * np.abs(g * u) + 1e-30
    kinds = [("dense", torch.float32), ("dense", torch.bfloat16), ("held", None), ("both", torch.bfloat16)]
    for kind, dtype in kinds:
        for keep in (False, True):
            h = Guarded(rows, f) if kind != "dense" else None
            y = torch.full((rows, f + 3), -3.0, dtype=dtype, device=DEV) if kind != "held" else None
            gate, up = (Guarded(rows, f), Guarded(rows, f)) if keep else (None, None)
            B.dct_gated8_fwd(put(x), put(wg), put(wu), B.DCT_ACT_GELU if gelu else B.DCT_ACT_SILU, h and h.a, y, f + 3,
                             gate and gate.a, up and up.a)
            if h:
                assert near_held(h.read(), act * u, off_h)
            if y is not None:
                assert (np.abs(f64(y)[:, :f] - act * u) <= off_h + HALF[dtype] * (np.abs(act * u) + off_h)).all()
                assert bool((y[:, f:] == -3.0).all())
            if keep:
                assert near_held(gate.read(), g, off_g) and near_held(up.read(), u, off_u)


def slopes(dh, gate, up, gelu):
    act, slope = o.activation(gate, gelu)
    return dh * up * slope, dh * act, act * up


@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,f,pad,offset", [(1, 1, 0, 0), (1, 300, 0, 0), (7, 128, 0, 0), (128, 128, 0, 0), (129, 520, 3, 1), (300, 257, 0, 0)])
def test_gated_backward(rows, f, pad, offset, dtype, gelu):
    gate, up = matrix(rows, f, 1), matrix(rows, f, 2)
    dh = rows_of(rows, f, dtype, 3, pad, offset)
    want = slopes(f64(dh)[:, :f], o.values(gate), o.values(up), gelu)
    # a product of three fp32 factors, the slope's own terms of a few times its size (|g act''| stays below 2.5)
    off = [2.0 ** -17 * np.abs(f64(dh)[:, :f] * o.values(up)) * 4, 2.0 ** -17 * np.abs(f64(dh)[:, :f] * o.values(gate)),
           2.0 ** -17 * np.abs(o.values(gate) * o.values(up))]
    forms = [(0, False), (1, False), (0, True), (1, True), (2, True)]
    for chosen in (range(5), (0,), (1,), (2,), (3,), (4,), (0, 1), (2, 3, 4)):
        out = [(Guarded(f, rows) if turned else Guarded(rows, f)) if i in chosen else None for i, (_, turned) in enumerate(forms)]
        B.dct_gated8_bwd(dh if set(chosen) != {4} else None, f + pad, put(gate), put(up), B.DCT_ACT_GELU if gelu else B.DCT_ACT_SILU,
                         *(m and m.a for m in out))
        for i in chosen:
            which, turned = forms[i]
            w, e = (want[which].T, off[which].T) if turned else (want[which], off[which])
            assert near_held(out[i].read(), w, e)


def test_gated_gradients_against_differences():
    """The slopes are the derivative of the forward block: (h(g + s) - h(g - s)) / 2s, all in values that 8 bits hold."""
    rows, f = 64, 256
    for gelu in (False, True):
        g = f64(torch.randn(rows, f, generator=gen(1), device=DEV) * 2)
        u = o.values(o.hold(f64(torch.randn(rows, f, generator=gen(2), device=DEV))))
        held = o.hold(g)
        g, s = o.values(held), 1e-4
        dg = Guarded(rows, f)
        ones = torch.ones(rows, f, device=DEV)
        B.dct_gated8_bwd(ones, f, put(held), put(o.hold(u)), int(gelu), dg.a)
        want = (o.activation(g + s, gelu)[0] - o.activation(g - s, gelu)[0]) / (2 * s) * u
        assert near_held(dg.read(), want, 1e-6 * np.abs(u) + 1e-9)


def test_products_of_codes_fall_on_the_right_side_of_a_border():
    """g u of two codes is often halfway between two codes, and act(g) u is just beside it: for large g the share is 1 in fp32 (and in
    64 bits), but never is."""
    rows, f = 128, 256
    g = np.tile(np.ldexp(1 + np.arange(8) / 8, 5), (rows, f // 8))           # 32 .. 60
    u = np.tile(np.repeat(1 + np.arange(8) / 8, 8), (rows, f // 64))
    p = g * u
    steps = np.ldexp(p, 3 - (np.frexp(p)[1] - 1))
    border = steps % 1 == 0.5
    assert border.any()
    for gelu in (False, True):
        h_t, dup = Guarded(f, rows), Guarded(rows, f)
        B.dct_gated8_bwd(torch.from_numpy(u).float().to(DEV), f, put(o.hold(g)), put(o.hold(u)), int(gelu), None, dup.a, None, None, h_t.a)
        for got in (o.values(h_t.read()).T, o.values(dup.read())):
            low = np.ldexp(np.floor(steps), np.frexp(p)[1] - 1 - 3)
            assert np.array_equal(got[border], low[border])


# ---- streams, graphs, sizes ----

def test_another_stream_and_repeated_calls():
    a, b, x = put(matrix(200, 900, 1)), put(matrix(300, 900, 2)), put(matrix(7, 900, 3))
    first = torch.empty(200, 300, device=DEV)
    few = torch.empty(7, 300, device=DEV)
    B.dct_gemm8(a, b, first, 300)
    B.dct_gemm8(x, b, few, 300)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        c, d = torch.empty_like(first), torch.empty_like(few)
        torch.cuda.synchronize()
        B.dct_gemm8(a, b, c, 300, stream=side)
        B.dct_gemm8(x, b, d, 300)                   # at the same time on the current one
        torch.cuda.synchronize()
        assert torch.equal(c, first) and torch.equal(d, few)


def ffn(x, dh, state):
    """The calls of a block, forward and backward, as a user makes them."""
    rows, d, f = x.shape[0], x.shape[1], state["wg"].rows
    B.dct_act8_pack(x, rows, d, d, state["x"], state["x_t"])
    B.dct_gated8_fwd(state["x"], state["wg"], state["wu"], B.DCT_ACT_SILU, state["h"], None, 0, state["gate"], state["up"])
    B.dct_gated8_bwd(dh, f, state["gate"], state["up"], B.DCT_ACT_SILU, state["dg"], state["du"], state["dg_t"], state["du_t"], state["h_t"])
    B.dct_gemm8(state["dg"], state["wg_t"], state["dx"], d, state["du"], state["wu_t"])
    B.dct_gemm8(state["dg_t"], state["x_t"], state["dwg"], d)


def ffn_state(rows, d, f, seed=0):
    g = gen(seed)
    s = {}
    for name in ("wg", "wu"):
        w = torch.randn(f, d, generator=g, device=DEV) * d ** -0.5
        s[name], s[name + "_t"] = B.new_act8(f, d), B.new_act8(d, f)
        B.dct_act8_pack(w, f, d, d, s[name], s[name + "_t"])
    s.update(x=B.new_act8(rows, d), x_t=B.new_act8(d, rows), dx=torch.empty(rows, d, device=DEV), dwg=torch.empty(f, d, device=DEV))
    for name in ("h", "gate", "up", "dg", "du"):
        s[name] = B.new_act8(rows, f)
    for name in ("dg_t", "du_t", "h_t"):
        s[name] = B.new_act8(f, rows)
    return s


@pytest.mark.parametrize("rows", [5, 300])
def test_captured_calls_are_replayed_and_two_graphs_run_at_once(rows):
    d, f = 260, 520
    xs = [torch.randn(rows, d, generator=gen(i), device=DEV, dtype=torch.float32).bfloat16() for i in range(2)]
    dhs = [torch.randn(rows, f, generator=gen(9 + i), device=DEV).bfloat16() for i in range(2)]
    states = [ffn_state(rows, d, f, i) for i in range(2)]
    want = []
    for x, dh, s in zip(xs, dhs, states):
        ffn(x, dh, s)
        want.append((s["dx"].clone(), s["dwg"].clone()))
    graphs = []
    for x, dh, s in zip(xs, dhs, states):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ffn(x, dh, s)
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for s in states:
            s["dx"].fill_(-1), s["dwg"].fill_(-1)
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for s, w in zip(states, want):
            assert torch.equal(s["dx"], w[0]) and torch.equal(s["dwg"], w[1])


def test_rows_whose_offset_passes_32_bits():
    """A checkpoint of over 4 GiB: its last rows are written, read, transposed and multiplied as by themselves."""
    cols, rows, last = 4096, (1 << 20) + 300, 40
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    x[-last:] = torch.randn(last, cols, generator=gen(1), device=DEV).bfloat16()
    big, small = B.new_act8(rows, cols), B.new_act8(last, cols)
    B.dct_act8_pack(x, rows, cols, cols, big)
    B.dct_act8_pack(x[-last:], last, cols, cols, small)
    assert torch.equal(big.codes[-last:], small.codes)
    del x
    y, z = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV), torch.empty(last, cols, dtype=torch.bfloat16, device=DEV)
    B.dct_act8_unpack(big, y, cols)
    B.dct_act8_unpack(small, z, cols)
    assert torch.equal(y[-last:], z) and not y[:-last].any()
    del y
    turned = B.new_act8(cols, rows)
    B.dct_act8_transpose(big, turned)
    back = B.new_act8(rows, cols)
    B.dct_act8_transpose(turned, back)
    y = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV)
    B.dct_act8_unpack(back, y, cols)
    assert not y[:-last].any()
    far = (y[-last:].float() - z.float()).abs()
    assert bool((far <= 2.0 ** -10 * z.abs().amax()).all())
    del y, back, turned
    w = put(matrix(96, cols, 7))
    c, e = torch.empty(rows, 96, device=DEV), torch.empty(last, 96, device=DEV)
    B.dct_gemm8(big, w, c, 96)
    B.dct_gemm8(small, w, e, 96)
    assert not c[:-last].any()
    assert bool(((c[-last:] - e).abs() <= 1e-4 * e.abs().amax()).all())


# ---- waits that run out, several threads, a first call inside a capture ----

def test_waits_that_run_out_lose_values_and_nothing_else():
    """With a limit of one look at a barrier most waits give up: what is written is then right or NaN, every call ends, and the next one (with
    the usual limit) is right."""
    x, w = rows_of(300, 700, torch.bfloat16, 1), rows_of(400, 700, torch.float32, 2)
    dh = rows_of(300, 400, torch.bfloat16, 3)
    big = rows_of(4000, 300, torch.bfloat16, 4)

    def calls():
        out = {}
        a, t, b = B.new_act8(300, 700), B.new_act8(700, 300), B.new_act8(400, 700)
        B.dct_act8_pack(x, 300, 700, 700, a, t)
        B.dct_act8_pack(w, 400, 700, 700, b)
        g = put(matrix(4000, 300, 5))
        turned = B.new_act8(300, 4000)
        B.dct_act8_transpose(g, turned)
        few, mid, pairs = (torch.empty(*size, device=DEV) for size in ((9, 400), (300, 400), (4000, 2600)))
        p, q = put(matrix(300, 700, 6)), put(matrix(400, 700, 7))
        B.dct_gemm8(put(matrix(9, 700, 8)), q, few, 400)
        B.dct_gemm8(p, q, mid, 400)
        B.dct_gemm8(g, put(matrix(2600, 300, 9)), pairs, 2600)
        wide, narrow = torch.empty(300, 400, device=DEV), torch.empty(9, 400, device=DEV)
        B.dct_gated8_fwd(p, q, put(matrix(400, 700, 10)), B.DCT_ACT_SILU, None, wide, 400)
        B.dct_gated8_fwd(put(matrix(9, 700, 8)), q, put(matrix(400, 700, 10)), B.DCT_ACT_SILU, None, narrow, 400)
        dg = B.new_act8(400, 300)
        kept = put(matrix(300, 400, 11))
        B.dct_gated8_bwd(dh, 400, kept, kept, B.DCT_ACT_SILU, dgate_t=dg)
        for name, m in (("a", a), ("t", t), ("turned", turned), ("dg", dg)):
            out[name] = torch.empty(m.rows, m.cols, device=DEV)
            B.dct_act8_unpack(m, out[name], m.cols)
        out.update(few=few, mid=mid, pairs=pairs, wide=wide, narrow=narrow)
        torch.cuda.synchronize()
        return out

    want = calls()
    try:
        B.dct_debug_configure(1, 0)
        for _ in range(3):
            got = calls()
            for name, v in got.items():
                assert bool((torch.isnan(v) | (v == want[name])).all()), name
    finally:
        B.dct_debug_configure()
    for name, v in calls().items():
        assert torch.equal(v, want[name]), name


def test_several_threads_call_at_once():
    import threading
    a, b = matrix(200, 600, 1), matrix(300, 600, 2)
    pa, pb = put(a), put(b)
    want = torch.empty(200, 300, device=DEV)
    B.dct_gemm8(pa, pb, want, 300)
    torch.cuda.synchronize()
    out, errors = [torch.empty_like(want) for _ in range(4)], []

    def work(i):
        try:
            stream = torch.cuda.Stream()
            for _ in range(50):
                out[i].fill_(-1.0)
                stream.wait_stream(torch.cuda.current_stream())
                B.dct_gemm8(pa, pb, out[i], 300, stream=stream)
                stream.synchronize()
                if not torch.equal(out[i], want):
                    errors.append(i)
        except Exception as e:           # (an exception in a thread would only be printed)
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors


def test_the_first_call_of_a_process_may_be_captured():
    import subprocess
    import sys
    code = """
import torch
from paper_2010_08899_b200 import binding as B
x = torch.randn(70, 256, device="cuda").bfloat16()
a, t, c, h = B.new_act8(70, 256), B.new_act8(256, 70), torch.empty(70, 70, device="cuda"), torch.empty(70, 70, device="cuda")
few, f = B.new_act8(5, 256), torch.empty(5, 70, device="cuda")
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    B.dct_act8_pack(x, 70, 256, 256, a, t)
    B.dct_act8_pack(x, 5, 256, 256, few)
    B.dct_gemm8(a, a, c, 70)
    B.dct_gemm8(few, a, f, 70)
    B.dct_gated8_fwd(a, a, a, B.DCT_ACT_SILU, None, h, 70)
graph.replay()
torch.cuda.synchronize()
y = torch.empty(70, 256, device="cuda")
B.dct_act8_unpack(a, y, 256)
want = (y.double() @ y.double().T)
assert (c.double() - want).abs().max() <= 1e-4 * want.abs().max()
assert torch.equal(f, c[:5]) or (f - c[:5]).abs().max() <= 1e-4 * want.abs().max()
assert torch.isfinite(h).all()
"""
    done = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]
