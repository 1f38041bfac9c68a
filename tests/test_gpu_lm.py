"""The layer norm and the calls on rows of logits on the GPU against the 64-bit oracle.

Tolerances, with u = 2^-24 (one rounding of fp32) and `chain(n)` = 4 sqrt(n / 64) the usual size of the error of an
fp32 sum of n terms in at least 64 chains, in roundings (four standard deviations of a random walk); 64 u stands for
the few roundings and the 2-ulp functions around it.  A bf16 result (8 significant bits) adds
half a step: up to 2^-8 of its size.
Whole numbers are compared exactly."""
import numpy as np
import pytest
import torch

from oracle import lm
from paper_2010_08899_b200 import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda"
U = 2.0 ** -24
GUARD = 64
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
FILL = 77.0


def chain(n):
    return 4.0 * np.sqrt(n / 64.0)


def f64(t):
    return t.detach().double().cpu().numpy()


def half_step(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else U


def matrix(rows, d, ld, offset, dtype, fill):
    """An uninitialised [rows, ld] matrix that starts ``offset`` elements past a 256-byte boundary, every element
    outside the first d columns of a row set to ``fill``; returns (whole buffer, flat view for the call, 2-D view)."""
    buf = torch.full((rows * ld + offset + 2 * GUARD,), fill, dtype=dtype, device=DEV)
    flat = buf[offset:offset + rows * ld]
    return buf, flat, flat.view(rows, ld)


def put(values, ld, offset):
    rows, d = values.shape
    buf, flat, view = matrix(rows, d, ld, offset, values.dtype, FILL)
    view[:, :d] = values.to(DEV)
    return flat


def only_rows_written(buf, flat, rows, d, ld, fill=FILL):
    """Every element outside the rows' first d columns still holds the fill."""
    probe = buf.clone()
    off = (flat.data_ptr() - buf.data_ptr()) // buf.element_size()
    probe[off:off + rows * ld].view(rows, ld)[:, :d] = fill
    return bool((probe == fill).all())


def vec(n, dtype=torch.float32, fill=FILL):
    return torch.full((n + GUARD,), fill, dtype=dtype, device=DEV)


def guard_ok(t, n, fill=FILL):
    return bool((t[n:] == fill).all())


def close(got, want, tol):
    """got within tol of want elementwise; infinities and NaN have to agree."""
    got, want = np.asarray(got), np.asarray(want)
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)])
    err = np.abs(got[fine] - want[fine])
    tol = np.broadcast_to(tol, want.shape)[fine]
    assert (err <= tol).all(), f"worst error {np.max(err - tol)} over its tolerance, at error {err[np.argmax(err - tol)]}"


# ----------------------------------------------------------------------------------------------------------------
# layer norm
# ----------------------------------------------------------------------------------------------------------------

NORM_SHAPES = [(1, 1, 1, 0), (3, 2, 2, 1), (5, 7, 9, 3), (33, 31, 31, 0), (4, 33, 40, 1), (257, 64, 64, 0), (70, 100, 100, 0),
               (19, 128, 136, 0), (301, 512, 512, 0), (45, 511, 511, 0), (45, 513, 520, 0), (23, 1000, 1001, 1),
               (9, 1024, 1024, 4), (700, 1536, 1536, 0), (31, 2047, 2047, 0), (17, 4096, 4096, 0), (13, 5003, 5003, 0),
               (11, 8192, 8192, 0), (6, 8193, 8200, 0), (5, 12288, 12288, 0), (4, 16384, 16384, 2), (3, 33000, 33000, 0),
               (2, 65536, 65536, 0)]


def norm_tolerances(x, w, b, o, d, dtype):
    r = o.rstd[:, None]
    h = (x - o.mean[:, None]) * r
    shift = (np.abs(x) + np.abs(o.mean)[:, None]) * r                    # what one rounding of x - mean is relative to
    ww = np.ones(d) if w is None else w
    bb = np.zeros(d) if b is None else b
    c = 64 + chain(d)
    tol_y = U * (c * (1 + np.abs(h)) + 4 * shift) * np.abs(ww) + U * 4 * np.abs(bb) + half_step(dtype) * np.abs(o.y)
    size = np.abs(x).mean(axis=1)
    # the mean is off by U c size; squared deviations see it in the second order, and their own roundings in the first
    return tol_y + U * c * (size * o.rstd)[:, None] * np.abs(ww), U * c * size, U * o.rstd * (c + 8 * (shift ** 2).mean(axis=1))


@pytest.mark.parametrize("rows,d,ld,offset", NORM_SHAPES)
@pytest.mark.parametrize("dtype,pdtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
def test_layer_norm(rows, d, ld, offset, dtype, pdtype):
    dt, pdt = DT[dtype], DT[pdtype]
    gen = torch.Generator().manual_seed(1000 + d)
    x = (torch.randn(rows, d, generator=gen) * torch.exp(torch.randn(rows, 1, generator=gen)) + 0.5).to(dt)
    dy = torch.randn(rows, d, generator=gen).to(dt)
    w = (1 + 0.3 * torch.randn(d, generator=gen)).to(pdt)
    b = (0.2 * torch.randn(d, generator=gen)).to(pdt)
    use_w, use_b = d % 3 != 1, d % 5 != 1
    eps = 1e-5
    xd, ow, ob = f64(x), f64(w) if use_w else None, f64(b) if use_b else None
    o = lm.layer_norm_fwd(xd, ow, ob, np.float32(eps).astype(np.float64))
    tol_y, tol_mean, tol_rstd = norm_tolerances(xd, ow, ob, o, d, dt)

    x_flat = put(x, ld, offset)
    ld_y = ld + (d % 2)
    y_buf, y_flat, y = matrix(rows, d, ld_y, offset, dt, FILL)
    mean, rstd = vec(rows), vec(rows)
    B.dct_layer_norm_fwd(x_flat, rows, d, ld, w.to(DEV) if use_w else None, b.to(DEV) if use_b else None, eps, y_flat, ld_y,
                         mean, rstd)
    close(f64(y[:, :d]), o.y, tol_y)
    close(f64(mean[:rows]), o.mean, tol_mean)
    close(f64(rstd[:rows]), o.rstd, tol_rstd)
    assert only_rows_written(y_buf, y_flat, rows, d, ld_y) and guard_ok(mean, rows) and guard_ok(rstd, rows)

    # backward from the numbers the forward call left
    mu, rs = f64(mean[:rows]), f64(rstd[:rows])
    dyd = f64(dy)
    want = lm.layer_norm_bwd(dyd, xd, ow, mu, rs)
    dy_flat = put(dy, ld_y, offset)
    dx_buf, dx_flat, dx = matrix(rows, d, ld, offset, dt, FILL)
    dw, db = vec(d), vec(d)
    ws = B.new_workspace(B.dct_layer_norm_bwd_workspace_bytes(rows, d))
    ws.fill_(0xFF)                                                       # NaN, should anything be read before it is written
    wt = w.to(DEV) if use_w else None
    B.dct_layer_norm_bwd(dy_flat, ld_y, x_flat, rows, d, ld, wt, mean[:rows], rstd[:rows], dx_flat, ld, dw, db, ws)
    h = (xd - mu[:, None]) * rs[:, None]
    shift = (np.abs(xd) + np.abs(mu)[:, None]) * rs[:, None]
    g = np.abs(dyd * (1.0 if ow is None else ow))
    c = 64 + chain(d)
    m2 = (g * (np.abs(h) + shift)).mean(axis=1, keepdims=True)
    tol_dx = U * rs[:, None] * (c * (g + g.mean(axis=1, keepdims=True)) + (c * np.abs(h) + 4 * shift) * m2) \
        + half_step(dt) * np.abs(want.dx)
    close(f64(dx[:, :d]), want.dx, tol_dx)
    cr = 64 + chain(rows)
    close(f64(dw[:d]), want.dweight, U * cr * (np.abs(dyd) * (np.abs(h) + shift)).sum(axis=0))
    close(f64(db[:d]), want.dbias, U * cr * np.abs(dyd).sum(axis=0))
    assert only_rows_written(dx_buf, dx_flat, rows, d, ld) and guard_ok(dw, d) and guard_ok(db, d)

    # the same bits again, in place of dy and of x, and without the parameters' gradients
    for place in ("dy", "x", "none"):
        dy2, x2 = put(dy, ld, offset), put(x, ld, offset)
        out = dy2 if place == "dy" else x2 if place == "x" else torch.empty_like(x2)
        dw2, db2 = (None, None) if place == "none" else (vec(d), vec(d))
        B.dct_layer_norm_bwd(dy2, ld, x2, rows, d, ld, wt, mean[:rows], rstd[:rows], out, ld, dw2, db2,
                             None if place == "none" else ws)
        assert torch.equal(out.view(rows, ld)[:, :d], dx[:, :d])
        if place != "none":
            assert torch.equal(dw2, dw) and torch.equal(db2, db)
    x2 = put(x, ld, offset)
    B.dct_layer_norm_fwd(x2, rows, d, ld, wt, b.to(DEV) if use_b else None, eps, x2, ld)
    assert torch.equal(x2.view(rows, ld)[:, :d], y[:, :d])


@pytest.mark.parametrize("d", [64, 1000, 4096, 9000])
def test_layer_norm_of_rows_far_from_zero(d):
    """A mean a thousand times the deviation: the variance comes from deviations, not from a difference of squares."""
    gen = torch.Generator().manual_seed(5)
    x = 1000.0 + torch.randn(8, d, generator=gen)
    o = lm.layer_norm_fwd(f64(x), None, None, float(np.float32(1e-5)))
    y, mean, rstd = torch.empty(8, d, device=DEV), vec(8), vec(8)
    B.dct_layer_norm_fwd(x.to(DEV), 8, d, d, None, None, 1e-5, y, d, mean, rstd)
    tol_y, tol_mean, _ = norm_tolerances(f64(x), None, None, o, d, torch.float32)
    close(f64(y), o.y, tol_y)
    close(f64(mean[:8]), o.mean, tol_mean)
    # the mean is off by up to delta = U c 1000: the variance by delta^2, far below a difference of squares' 1000^2 U
    delta = U * (64 + chain(d)) * 1000.0
    close(f64(rstd[:8]), o.rstd, o.rstd * (U * (64 + chain(d)) + delta ** 2 + 4 * U * 1000.0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layer_norm_empty_constant_and_broken_rows(dtype):
    dt = DT[dtype]
    for d in (48, 1000):
        x = torch.randn(6, d, generator=torch.Generator().manual_seed(3)).to(dt)
        x[1], x[2, 3], x[3, 4] = 2.5, float("nan"), float("inf")
        y, mean, rstd = torch.empty(6, d, dtype=dt, device=DEV), vec(6), vec(6)
        B.dct_layer_norm_fwd(x.to(DEV), 6, d, d, None, None, 1e-5, y, d, mean, rstd)
        assert bool((y[1] == 0).all()) and float(mean[1]) == 2.5
        assert bool(y[2:4].isnan().all()) and bool(y[0].isfinite().all()) and bool(y[4:].isfinite().all())
    e = torch.empty(0, dtype=dt, device=DEV)
    f = torch.empty(0, device=DEV)
    B.dct_layer_norm_fwd(e, 0, 16, 16, None, None, 1e-5, e, 16, f, f)
    dw, db = vec(16), vec(16)
    B.dct_layer_norm_bwd(e, 16, e, 0, 16, 16, None, f, f, e, 16, dw, db, B.new_workspace(256))
    assert not dw[:16].any() and not db[:16].any() and guard_ok(dw, 16) and guard_ok(db, 16)


# ----------------------------------------------------------------------------------------------------------------
# log-probabilities
# ----------------------------------------------------------------------------------------------------------------

LP_SHAPES = [(1, 1, 1, 0, 1), (2, 2, 3, 1, 2), (5, 7, 7, 0, 7), (9, 31, 31, 1, 5), (4, 64, 64, 0, 64), (33, 100, 104, 0, 20),
             (3, 255, 255, 2, 128), (7, 1000, 1000, 0, 256), (6, 1023, 1027, 3, 17), (40, 4096, 4096, 0, 1),
             (12, 5003, 5003, 0, 64), (3, 10007, 10007, 1, 16), (300, 2050, 2050, 0, 8), (2, 32768, 32768, 0, 100),
             (5, 50021, 50021, 0, 20), (1, 131072, 131072, 0, 20), (2, 151001, 151008, 5, 256), (160, 16392, 16392, 0, 33),
             (1, 1048576, 1048576, 0, 50), (3, 262145, 262145, 0, 7)]


def logits(rows, vocab, seed, dtype):
    gen = torch.Generator().manual_seed(seed)
    x = 2.5 * torch.randn(rows, vocab, generator=gen)
    peak = torch.randint(0, vocab, (rows,), generator=gen)
    x[torch.arange(rows), peak] += torch.rand(rows, generator=gen) * 14
    return x.to(dtype), peak


def check_logprobs(x, inv_t, tokens, top, ld, offset, dt, want_result=True, stream=None):
    rows, vocab = x.shape
    flat = put(x, ld, offset)
    lp, ent, stats = vec(rows), vec(rows), vec(2 * rows)
    ids, tlp = vec(rows * top, torch.int32, -7), vec(rows * top)
    res = B.new_result() if want_result else None
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    B.dct_lm_logprobs_fwd(flat, rows, vocab, ld, inv_t, tokens.to(DEV), top, lp, ent, stats, ids if top else None,
                          tlp if top else None, res, stream=stream)
    if stream is not None:
        torch.cuda.current_stream().wait_stream(stream)
    xd = f64(x)
    o = lm.log_probs(xd, float(np.float32(inv_t)))
    tok = tokens.numpy()
    ok = (tok >= 0) & (tok < vocab)
    c = U * (64 + chain(vocab))
    live = o.max > -np.inf
    mag = np.where(np.isfinite(o.max), np.abs(o.max), 0.0)
    tol_s = c * (1 + np.abs(np.nan_to_num(o.logsum))) + 2 * U * mag
    want_lp = np.where(ok, o.logp[np.arange(rows), np.where(ok, tok, 0)], 0.0)
    size = lambda v: np.where(np.isfinite(v), np.abs(v), 0.0)
    close(f64(lp[:rows]), want_lp, tol_s + 8 * U * size(want_lp))
    # the entropy is a sum of terms p |log p| and of the logarithm; a reference up to 16 binades off costs no more than 12 of them
    close(f64(ent[:rows]), o.entropy, (c + 16 * U) * (12 + np.nan_to_num(o.entropy)) + 2 * U * mag)
    got = f64(stats[:2 * rows]).reshape(rows, 2)
    close(got[:, 0], o.max, 2 * U * mag)
    close(got[:, 1], o.logsum, tol_s)
    if top:
        want_ids = np.stack([lm.top_columns(xd[i], top) for i in range(rows)])
        assert np.array_equal(ids[:rows * top].cpu().numpy().reshape(rows, top), want_ids)
        want_t = np.take_along_axis(o.logp, want_ids.astype(np.int64), 1)
        close(f64(tlp[:rows * top]).reshape(rows, top), want_t, tol_s[:, None] + 8 * U * size(want_t))
    assert guard_ok(lp, rows) and guard_ok(ent, rows) and guard_ok(stats, 2 * rows)
    assert guard_ok(ids, rows * top, -7) and guard_ok(tlp, rows * top)
    if want_result:
        assert B.read_result(res).status == (B.DCT_ERR_BAD_MASK if (tok >= vocab).any() else B.DCT_OK)
    return flat, stats[:2 * rows], ent[:rows], o


@pytest.mark.parametrize("rows,vocab,ld,offset,top", LP_SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logprobs_forward_and_backward(rows, vocab, ld, offset, top, dtype):
    dt = DT[dtype]
    inv_t = (1.0, 0.7, 1.5)[vocab % 3]
    x, peak = logits(rows, vocab, 2000 + vocab, dt)
    tokens = peak.to(torch.int32)
    tokens[rows // 2] = (tokens[rows // 2] + 1) % vocab
    if rows > 2:
        tokens[1], tokens[2] = -1, vocab            # nothing asked; a token outside the vocabulary
    flat, stats, ent, o = check_logprobs(x, inv_t, tokens, top, ld, offset, dt, want_result=rows != 5)

    gen = torch.Generator().manual_seed(7)
    a, c = torch.randn(rows, generator=gen), torch.randn(rows, generator=gen)
    st = f64(stats).reshape(rows, 2)
    for use_a, use_c in ((True, True), (True, False), (False, True)):
        want = lm.log_probs_bwd(f64(x), float(np.float32(inv_t)), tokens.numpy(), st[:, 0], st[:, 1], f64(ent),
                                f64(a) if use_a else None, f64(c) if use_c else None)
        g_buf, g_flat, g = matrix(rows, vocab, ld, offset, dt, FILL)
        B.dct_lm_logprobs_bwd(flat, rows, vocab, ld, inv_t, tokens.to(DEV) if use_a else None, stats,
                              ent if use_c else None, a.to(DEV) if use_a else None, c.to(DEV) if use_c else None, g_flat, ld)
        lp = f64(x) * float(np.float32(inv_t)) - st.sum(axis=1, keepdims=True)
        p = np.exp(lp)
        aa, cc = f64(a)[:, None] * use_a, f64(c)[:, None] * use_c
        big = np.abs(st).sum(axis=1, keepdims=True)
        rel = U * (32 + 8 * np.abs(lp) + 4 * big)
        tol = inv_t * (rel * p * (np.abs(aa) + np.abs(cc) * (1 + np.abs(lp) + f64(ent)[:, None]))) \
            + half_step(dt) * np.abs(want) * 1.01
        hit = (tokens.numpy() >= 0) & (tokens.numpy() < vocab)
        tol[hit, tokens.numpy()[hit]] += inv_t * 4 * U * np.abs(f64(a)[hit]) * use_a
        close(f64(g[:, :vocab]), want, tol + 1e-37)
        assert only_rows_written(g_buf, g_flat, rows, vocab, ld)
        if use_a and use_c:
            again = flat.clone()
            in_place = put(x, ld, offset)
            B.dct_lm_logprobs_bwd(in_place, rows, vocab, ld, inv_t, tokens.to(DEV), stats, ent, a.to(DEV), c.to(DEV), in_place, ld)
            assert torch.equal(in_place.view(rows, ld)[:, :vocab], g[:, :vocab])
            other = torch.empty(rows * (vocab + 3), dtype=dt, device=DEV)
            B.dct_lm_logprobs_bwd(flat, rows, vocab, ld, inv_t, tokens.to(DEV), stats, ent, a.to(DEV), c.to(DEV), other, vocab + 3)
            assert torch.equal(other.view(rows, vocab + 3)[:, :vocab], g[:, :vocab]) and torch.equal(again, flat)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [3, 70, 1000, 4099, 40000])
def test_logprobs_of_masked_and_broken_rows(dtype, vocab):
    dt = DT[dtype]
    low = torch.finfo(dt).min
    inf, nan = float("inf"), float("nan")
    top = min(vocab, 60)
    x, peak = logits(14, vocab, 31, dt)
    x[0] = -inf                                        # nothing left
    x[1] = -inf
    x[1, vocab // 2] = 1.5                             # one column left
    x[2] = low                                         # the lowest value throughout: uniform
    x[3, 1:] = low                                     # masked by the lowest value
    x[4] = 3.0                                         # all equal
    x[5] = torch.where(torch.arange(vocab) % 2 == 0, 0.0, -0.0).to(dt)
    x[6, vocab - 1] = inf
    x[7, 0] = nan
    x[8] = nan
    x[9] = -nan
    x[10] = torch.where(torch.arange(vocab) % 3 == 0, x[10], torch.tensor(-inf, dtype=dt))
    x[11] = torch.arange(vocab).to(dt) * 0.25          # sorted, with runs of equal values in bf16
    x[12] = -torch.arange(vocab).to(dt) * 0.25
    x[13, :] = nan
    x[13, vocab // 3] = -inf
    tokens = torch.full((14,), vocab - 1, dtype=torch.int32)
    flat, stats, ent, o = check_logprobs(x, 1.0, tokens, top, vocab, 0, dt)
    a = torch.ones(14)
    g = torch.empty(14 * vocab, dtype=dt, device=DEV)
    B.dct_lm_logprobs_bwd(flat, 14, vocab, vocab, 1.0, tokens.to(DEV), stats, ent, a.to(DEV), a.to(DEV), g, vocab)
    g = f64(g).reshape(14, vocab)
    assert not g[0].any()                              # no distribution: no gradient
    assert np.isfinite(g[[1, 2, 3, 4, 5, 10, 11, 12]]).all()
    for i in (6, 7, 8, 9):
        assert np.isnan(g[i]).any()
    assert abs(g[4].sum()) <= vocab * (2.0 ** -8 / vocab + U)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,top", [(5000, 5), (40000, 256), (300000, 64)])
def test_top_of_rows_with_many_equal_values(dtype, vocab, top):
    """A few distinct values only, fewer large ones than asked for, the large ones in one stretch, all in one place."""
    dt = DT[dtype]
    gen = torch.Generator().manual_seed(11)
    x = torch.randint(0, 3, (7, vocab), generator=gen).float()
    x[1] = (torch.rand(vocab, generator=gen) < 2.0 * top / vocab).float()
    x[2] = 0.0
    x[2, vocab // 2:vocab // 2 + 2 * top] = 1.0 + torch.arange(2 * top) % 7
    x[3] = torch.randn(vocab, generator=gen)
    x[3, vocab - top // 2:] = 50.0
    x[4] = torch.randn(vocab, generator=gen).round(decimals=1)
    x[5] = torch.linspace(-3, 3, vocab)
    x[6] = torch.linspace(3, -3, vocab)
    check_logprobs(x.to(dt), 1.0, torch.zeros(7, dtype=torch.int32), top, vocab, 0, dt)


def test_logprobs_outputs_are_optional_and_follow_the_stream():
    x, peak = logits(6, 3001, 41, torch.float32)
    tokens = peak.to(torch.int32)
    side = torch.cuda.Stream()
    check_logprobs(x, 1.0, tokens, 9, 3001, 0, torch.float32, stream=side)
    xd = x.to(DEV).reshape(-1)
    full = [vec(6), vec(6), vec(12), vec(6 * 9, torch.int32), vec(6 * 9)]
    B.dct_lm_logprobs_fwd(xd, 6, 3001, 3001, 1.0, tokens.to(DEV), 9, *full)
    ent, stats, ids, tlp = vec(6), vec(12), vec(6 * 9, torch.int32), vec(6 * 9)
    B.dct_lm_logprobs_fwd(xd, 6, 3001, 3001, 1.0, None, 0, None, ent)
    B.dct_lm_logprobs_fwd(xd, 6, 3001, 3001, 1.0, None, 0, None, None, stats)
    B.dct_lm_logprobs_fwd(xd, 6, 3001, 3001, 1.0, None, 9, None, None, None, ids, tlp)
    for got, want in zip((ent, stats, ids, tlp), full[1:]):
        assert torch.equal(got, want)
    e = torch.empty(0, device=DEV)
    res = B.new_result()
    res.fill_(-1)
    B.dct_lm_logprobs_fwd(e, 0, 3001, 3001, 1.0, torch.empty(0, dtype=torch.int32, device=DEV), 0, e, e, e, result=res)
    B.dct_lm_logprobs_bwd(e, 0, 3001, 3001, 1.0, None, e, None, None, None, e, 3001)
    assert B.read_result(res).status == B.DCT_OK


# ----------------------------------------------------------------------------------------------------------------
# distillation
# ----------------------------------------------------------------------------------------------------------------

DS_SHAPES = [(1, 1, 1, 0, 1), (3, 2, 2, 1, 2), (6, 33, 35, 0, 5), (17, 100, 100, 3, 100), (9, 1000, 1000, 0, 64),
             (70, 1023, 1023, 1, 16), (11, 4096, 4096, 0, 32), (5, 10007, 10007, 0, 16), (3, 32768, 32768, 0, 64),
             (4, 50021, 50028, 0, 300), (2, 131072, 131072, 0, 128), (300, 2056, 2056, 0, 1024), (1, 300001, 300001, 1, 20),
             (1, 1048576, 1048576, 0, 1024)]


def teacher_of(x, top, seed, inv_t):
    rows, vocab = x.shape
    gen = torch.Generator().manual_seed(seed)
    z = x.float() * inv_t + 0.7 * torch.randn(rows, vocab, generator=gen)
    v, i = torch.topk(z, min(top, vocab), dim=1)
    lp = v - torch.logsumexp(z, 1, keepdim=True)
    ids = torch.full((rows, top), -1, dtype=torch.int32)
    t = torch.zeros(rows, top)
    ids[:, :v.shape[1]], t[:, :v.shape[1]] = i.to(torch.int32), lp
    return ids, t


def check_distill(x, inv_t, ids, t, tail, scale, ld, offset, dt):
    rows, vocab = x.shape
    top = ids.shape[1]
    mode = B.DCT_DISTILL_TAIL if tail else B.DCT_DISTILL_RENORM
    flat = put(x, ld, offset)
    loss = vec(rows)
    g_buf, g_flat, g = matrix(rows, vocab, ld, offset, dt, FILL)
    res = B.new_result()
    dev = lambda v: None if v is None else v.to(DEV)
    call = lambda src, out, ldo, lo: B.dct_lm_distill(src, rows, vocab, ld, inv_t, dev(ids), dev(t), top, mode, dev(scale),
                                                      lo, out, ldo, res)
    call(flat, g_flat, ld, loss)
    inv = float(np.float32(inv_t))
    xd, idn, td = f64(x), ids.numpy(), f64(t)
    o = lm.distill(xd, inv, idn, td, tail, None if scale is None else f64(scale))
    # sizes for the tolerances
    lp = lm.log_probs(xd, inv)
    c = U * (64 + chain(vocab) + chain(64 * top))
    valid = (idn >= 0) & (idn < vocab)
    tt = np.where(valid, td, -np.inf)
    if not tail:
        with np.errstate(invalid="ignore", divide="ignore"):
            tt = tt - tt.max(axis=1, keepdims=True)
            tt = tt - np.log(np.exp(tt).sum(axis=1, keepdims=True))
    q = np.nan_to_num(np.exp(tt))
    named = np.zeros((rows, vocab), dtype=bool)
    mass = np.zeros((rows, vocab))
    for i in range(rows):
        named[i, idn[i][valid[i]]] = True
        np.add.at(mass[i], idn[i][valid[i]], q[i][valid[i]])
    p = np.nan_to_num(np.exp(lp.logp))
    p_r = np.where(named, 0.0, p).sum(axis=1)
    q_r = np.maximum(0.0, 1.0 - q.sum(axis=1)) * tail
    with np.errstate(divide="ignore", invalid="ignore"):
        terms = q * (np.abs(np.nan_to_num(tt, neginf=0)) + np.abs(np.nan_to_num(
            np.take_along_axis(lp.logp, np.clip(idn, 0, vocab - 1).astype(np.int64), 1), neginf=0)))
        ratio = np.where((q_r > 0) & (p_r > 0), np.abs(np.log(q_r) - np.log(p_r)), 0.0)
    mag = np.where(np.isfinite(lp.max), np.abs(lp.max), 0.0)
    tol_loss = (c + 4 * U * mag) * (2 + terms.sum(axis=1)) + c * (ratio + 1) * tail
    close(f64(loss[:rows]), o.loss, tol_loss)
    s = (np.ones(rows) if scale is None else np.abs(f64(scale)))[:, None] * inv
    lpa = np.where(np.isfinite(lp.logp), np.abs(lp.logp), 0.0)
    rel = c + U * (8 * lpa + 4 * mag[:, None])
    share = np.where(named | (p_r[:, None] == 0), 0.0, p / np.where(p_r == 0, 1.0, p_r)[:, None])
    tol = s * (rel * (p + mass + share * q_r[:, None]) + (c + U * 8 * lpa) * mass + share * c * tail) \
        + half_step(dt) * 1.01 * np.abs(np.nan_to_num(o.grad)) + 1e-37
    close(f64(g[:, :vocab]), o.grad, tol)
    assert only_rows_written(g_buf, g_flat, rows, vocab, ld) and guard_ok(loss, rows)
    assert B.read_result(res).status == (B.DCT_ERR_BAD_MASK if (idn >= vocab).any() else B.DCT_OK)
    # the same bits with the loss alone, the gradient alone, another stride, and in place
    loss2 = vec(rows)
    call(flat, None, 0, loss2)
    assert torch.equal(loss2.view(torch.int32), loss.view(torch.int32))
    other = torch.empty(rows * (vocab + 1), dtype=dt, device=DEV)
    call(flat, other, vocab + 1, None)
    bits = torch.int32 if dt == torch.float32 else torch.int16
    assert torch.equal(other.view(rows, vocab + 1)[:, :vocab].contiguous().view(bits), g[:, :vocab].contiguous().view(bits))
    call(flat, flat, ld, loss2)
    assert torch.equal(flat.view(rows, ld)[:, :vocab].contiguous().view(bits), g[:, :vocab].contiguous().view(bits))
    return o


@pytest.mark.parametrize("rows,vocab,ld,offset,top", DS_SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tail", [False, True])
def test_distill(rows, vocab, ld, offset, top, dtype, tail):
    dt = DT[dtype]
    inv_t = (1.0, 0.5, 1.25)[vocab % 3]
    x, _ = logits(rows, vocab, 3000 + vocab, dt)
    ids, t = teacher_of(x, top, 5, inv_t)
    gen = torch.Generator().manual_seed(9)
    scale = None if rows == 9 else torch.rand(rows, generator=gen) * 2 - 0.5
    if rows > 2:
        ids[0, 0] = -1                                # an empty slot
        ids[1, top - 1] = vocab + 3                   # outside the vocabulary
        if top > 3:
            ids[2, 3] = ids[2, 1]                     # a column named twice
            t[2, 3] = t[2, 1] - 0.5
        perm = torch.randperm(top, generator=gen)     # slots in any order
        ids, t = ids[:, perm].contiguous(), t[:, perm].contiguous()
    check_distill(x, inv_t, ids, t, tail, scale, ld, offset, dt)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("vocab", [9, 1000, 40003])
def test_distill_of_degenerate_rows(dtype, tail, vocab):
    dt = DT[dtype]
    inf, nan = float("inf"), float("nan")
    top = 8
    x, _ = logits(16, vocab, 51, dt)
    ids, t = teacher_of(x, top, 6, 1.0)
    x[0] = -inf                                        # the student has nothing
    x[1, ids[1, 0]] = -inf                             # the teacher wants what the student cannot give
    ids[2] = -1                                        # the teacher says nothing
    t[3] = -inf                                        # slots without weight
    t[4, 2] = -inf
    x[5, 1] = nan
    x[6, 1] = inf
    t[7, 0] = nan
    x[8] = torch.finfo(dt).min                         # the lowest value throughout
    x[9] = -inf
    x[9, ids[9].long()] = torch.arange(top).to(dt)     # only named columns left: no remainder
    x[10] = -inf
    x[10, (ids[10, 0].long() + 1) % vocab] = 1.0
    x[11, ids[11].long()] = 90.0                       # a remainder of e^-90
    ids[12] = ids[12, 0]                               # one column in all slots
    t[13] = 0.0                                        # more than all of the mass (TAIL: no remainder)
    x[14, ids[14].long()] = -inf
    ids[15, 4:] = -1
    check_distill(x, 1.0, ids, t, tail, torch.linspace(0.5, 1.5, 16), vocab, 0, dt)
    # rows = 0
    e, i0 = torch.empty(0, dtype=dt, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    f = torch.empty(0, device=DEV)
    B.dct_lm_distill(e, 0, vocab, vocab, 1.0, i0, f, top, B.DCT_DISTILL_TAIL if tail else B.DCT_DISTILL_RENORM, None, f, e, vocab)


def test_distill_gradient_against_differences_of_the_loss():
    """The kernel's own loss, differenced at a few columns in fp32: steps of 2^-5 give a truncation error of
    step^2 / 6 (third derivatives of a softmax are below 1/4) and a rounding error of a few u |loss| / step."""
    rows, vocab, top, step = 4, 600, 12, 2.0 ** -5
    x, _ = logits(rows, vocab, 61, torch.float32)
    ids, t = teacher_of(x, top, 8, 1.0)
    dev = (ids.to(DEV), t.to(DEV))
    for mode in (B.DCT_DISTILL_RENORM, B.DCT_DISTILL_TAIL):
        g, loss = torch.empty(rows, vocab, device=DEV), torch.empty(rows, device=DEV)
        B.dct_lm_distill(x.to(DEV), rows, vocab, vocab, 1.0, *dev, top, mode, None, loss, g, vocab)
        scale = float(loss.abs().max())
        for j in list(ids[0, :4].tolist()) + [0, 17, 599]:
            ends = []
            for sign in (1.0, -1.0):
                y = x.clone()
                y[:, j] += sign * step
                out = torch.empty(rows, device=DEV)
                B.dct_lm_distill(y.to(DEV), rows, vocab, vocab, 1.0, *dev, top, mode, None, out)
                ends.append(out.double())
            slope = ((ends[0] - ends[1]) / (2 * step)).cpu().numpy()
            close(f64(g[:, j]), slope, step * step / 24 * 2 + U * (64 + chain(vocab)) * (8 + scale) / step)


# ----------------------------------------------------------------------------------------------------------------
# all of it together, graphs, and long matrices
# ----------------------------------------------------------------------------------------------------------------

def test_calls_can_be_captured_and_replayed():
    rows, vocab, top, d = 5, 9001, 10, 768
    x, peak = logits(rows, vocab, 71, torch.bfloat16)
    x, tokens = x.to(DEV).reshape(-1), peak.to(torch.int32).to(DEV)
    lp, ent, stats = vec(rows), vec(rows), vec(2 * rows)
    ids, tlp, loss = vec(rows * top, torch.int32), vec(rows * top), vec(rows)
    g, res = torch.empty(rows * vocab, dtype=torch.bfloat16, device=DEV), B.new_result()
    h, y = torch.randn(rows, d, device=DEV), torch.empty(rows, d, device=DEV)
    mean, rstd, dw, db = vec(rows), vec(rows), vec(d), vec(d)
    ws = B.new_workspace(B.dct_layer_norm_bwd_workspace_bytes(rows, d))

    def step():
        B.dct_layer_norm_fwd(h, rows, d, d, None, None, 1e-5, y, d, mean, rstd)
        B.dct_lm_logprobs_fwd(x, rows, vocab, vocab, 1.0, tokens, top, lp, ent, stats, ids, tlp, res)
        B.dct_lm_distill(x, rows, vocab, vocab, 0.5, ids[:rows * top], tlp[:rows * top], top, B.DCT_DISTILL_TAIL, None, loss, g, vocab, res)
        B.dct_layer_norm_bwd(y, d, h, rows, d, d, None, mean, rstd, y, d, dw, db, ws)

    step()
    torch.cuda.synchronize()
    outs = (lp, ent, stats, ids, tlp, loss, g, y, dw, db)
    want = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    for t in outs:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for got, ref in zip(outs, want):
        assert torch.equal(got[:ref.numel() - GUARD] if got.dim() == 1 and got is not g else got,
                           ref[:ref.numel() - GUARD] if got.dim() == 1 and got is not g else ref)


def test_offsets_beyond_32_bits():
    """A matrix of more than 2^32 elements: the last rows give what they give alone."""
    vocab, rows = 1 << 20, 4100
    x = torch.empty(rows * vocab, dtype=torch.bfloat16, device=DEV)
    x.zero_()
    tail, peak = logits(3, vocab, 81, torch.bfloat16)
    x[(rows - 3) * vocab:] = tail.to(DEV).reshape(-1)
    ids, t = teacher_of(tail, 20, 4, 1.0)
    all_ids, all_t = torch.zeros(rows, 20, dtype=torch.int32, device=DEV), torch.zeros(rows, 20, device=DEV)
    all_ids[-3:], all_t[-3:] = ids.to(DEV), t.to(DEV)
    small = tail.to(DEV).reshape(-1)
    for at, src, n in ((0, x, rows), (1, small, 3)):
        ent, stats, tid, tlp, loss = vec(n), vec(2 * n), vec(20 * n, torch.int32), vec(20 * n), vec(n)
        B.dct_lm_logprobs_fwd(src, n, vocab, vocab, 1.0, None, 20, None, ent, stats, tid, tlp)
        use_ids, use_t = (all_ids, all_t) if at == 0 else (ids.to(DEV), t.to(DEV))
        B.dct_lm_distill(src, n, vocab, vocab, 1.0, use_ids, use_t, 20, B.DCT_DISTILL_RENORM, None, loss, src, vocab)
        got = (ent[n - 3:n], stats[2 * n - 6:2 * n], tid[20 * n - 60:20 * n], tlp[20 * n - 60:20 * n], loss[n - 3:n],
               src[(n - 3) * vocab:n * vocab])
        if at == 0:
            big = [v.clone() for v in got]
    assert torch.equal(big[2], got[2])
    for a, b in zip(big, got):
        # one row's sums may be split over another number of blocks
        assert torch.allclose(a.double(), b.double(), rtol=2.0 ** -7, atol=1e-4 if a.numel() < 100 else 1e-9)
