"""Further edges of the layer norm and of the calls on rows of logits: masks, widths and shapes at which a choice of
kernel or of arithmetic changes.  Tolerances as in test_gpu_lm.py."""
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import lm
from paper_2010_08899_b200 import binding as B

from . import test_gpu_lm as base
from .conftest import ROOT
from .test_gpu_lm import DEV, DT, U, chain, check_distill, check_logprobs, close, f64, half_step, logits, vec

pytestmark = pytest.mark.gpu


def bits(t):
    return t.contiguous().view(torch.int32 if t.dtype == torch.float32 else torch.int16)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype,vocab,rows,top", [("f32", 1500, 300, 8), ("f32", 4000, 300, 8), ("f32", 6000, 300, 8),
                                                  ("f32", 10007, 300, 8), ("f32", 16000, 300, 8), ("bf16", 9001, 300, 8),
                                                  ("bf16", 32768, 230, 1024), ("bf16", 40003, 12, 8)])
def test_distill_of_lowest_rows_in_place(dtype, vocab, rows, top, tail):
    """Rows that hold the type's lowest value wherever a sum looks, with the gradient in the logits' place: CTAs of 1, 2, 4 and
    8 warps, rows that are loaded twice, and clusters.  Even rows are masked throughout (p = 1 / vocab); in odd ones the named
    columns alone are live (TAIL: none of them is streamed)."""
    dt = DT[dtype]
    gen = torch.Generator().manual_seed(vocab)
    x = torch.full((rows, vocab), torch.finfo(dt).min, dtype=dt)
    ids = torch.stack([torch.randperm(vocab, generator=gen)[:top] for _ in range(rows)]).to(torch.int32)
    live = torch.randn(rows, top, generator=gen).to(dt)
    odd = torch.arange(rows) % 2 == 1
    x[odd] = x[odd].scatter(1, ids[odd].long(), live[odd])
    t = torch.log_softmax(torch.randn(rows, top, generator=gen), 1) - 0.25
    mode = B.DCT_DISTILL_TAIL if tail else B.DCT_DISTILL_RENORM
    src, ids_d, t_d = x.to(DEV).reshape(-1), ids.to(DEV), t.to(DEV)
    apart, loss = torch.empty_like(src), vec(rows)
    B.dct_lm_distill(src, rows, vocab, vocab, 1.0, ids_d, t_d, top, mode, None, loss, apart, vocab)
    for _ in range(3):
        place, loss2 = src.clone(), vec(rows)
        B.dct_lm_distill(place, rows, vocab, vocab, 1.0, ids_d, t_d, top, mode, None, loss2, place, vocab)
        assert torch.equal(bits(place), bits(apart)) and torch.equal(bits(loss2), bits(loss))
    # the masked rows against the formula: equal logits are a uniform distribution, whatever they are
    even = (~odd).numpy()
    o = lm.distill(np.zeros((int(even.sum()), vocab)), 1.0, ids.numpy()[even], f64(t)[even], tail, None)
    c = U * (64 + chain(vocab) + chain(64 * top) + 8 * np.log(vocab))
    size = np.abs(f64(t)).max() + np.log(vocab)
    close(f64(loss[:rows])[even], o.loss, c * (2 + 4 * size))
    q = np.zeros((rows, vocab))
    np.put_along_axis(q, ids.numpy().astype(np.int64), np.exp(f64(t)), 1)
    close(f64(apart).reshape(rows, vocab)[even], o.grad, c * (4 / vocab + 4 * q[even]) + half_step(dt) * 1.01 * np.abs(o.grad))


def masked_rows(rows, vocab, fill, dt, seed):
    """Logits masked by a finite value in several manners, row by row in turn, and which rows hold nothing above it."""
    x, _ = logits(rows, vocab, seed, dt)
    fill = torch.tensor(fill).to(dt)
    col = torch.arange(vocab)
    gen = torch.Generator().manual_seed(seed + 1)
    for i in range(rows):
        kind = i % 7
        if kind == 0:
            x[i] = fill                                                      # throughout
        elif kind == 1:
            x[i, :vocab // 2] = fill                                         # what is read first
        elif kind == 2:
            x[i, :vocab - 2] = fill                                          # all but the last two
        elif kind == 3:
            x[i, 2:] = fill
        elif kind == 4:
            x[i] = torch.where((torch.rand(vocab, generator=gen) < 0.1) | (col == 1), x[i], fill)
        elif kind == 5:
            x[i] = torch.where(col % 3 == 0, fill, torch.tensor(float("-inf"), dtype=dt))      # a mask upon a mask
        else:
            x[i, vocab // 3:] = fill
    return x, torch.tensor([i % 7 in (0, 5) for i in range(rows)])


def from_their_largest(x):
    """The same distributions with the rows' largest value at 0 where it is far off."""
    top = x.max(axis=1, keepdims=True)
    with np.errstate(invalid="ignore"):
        return np.where(np.isfinite(top) & (top < -1e9), x - top, x)


FILLS = ["lowest", -1e10, -1e30]
FAR_SHAPES = [(7, 70, 7), (210, 1000, 20), (420, 4099, 9), (7, 40003, 20), (7, 200001, 5)]


@pytest.mark.parametrize("rows,vocab,top", FAR_SHAPES)
@pytest.mark.parametrize("inv_t", [1.0, 0.5, 0.6])
@pytest.mark.parametrize("fill", FILLS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logprobs_of_finite_masks(dtype, fill, inv_t, rows, vocab, top):
    dt = DT[dtype]
    x, whole = masked_rows(rows, vocab, torch.finfo(dt).min if fill == "lowest" else fill, dt, vocab)
    tokens = torch.arange(rows, dtype=torch.int32) * 7919 % vocab
    tokens[whole] -= tokens[whole] % 3                                       # (a column that the mask upon the mask leaves)
    flat, stats, ent, _ = check_logprobs(x, inv_t, tokens, top, vocab, 0, dt)
    # rows that the mask covers, against the uniform distribution they are
    lp, ids, tlp = vec(rows), vec(rows * top, torch.int32), vec(rows * top)
    B.dct_lm_logprobs_fwd(flat, rows, vocab, vocab, inv_t, tokens.to(DEV), top, lp, None, None, ids, tlp)
    inv, w = float(np.float32(inv_t)), whole.numpy()
    xs = from_their_largest(f64(x))
    o = lm.log_probs(xs, inv)
    c = U * (64 + chain(vocab))
    tol = c * (1 + np.abs(o.logsum))[w]
    want = o.logp[np.arange(rows), tokens.numpy()]
    close(f64(lp[:rows])[w], want[w], tol + 8 * U * np.abs(want[w]))
    close(f64(ent)[w], o.entropy[w], (c + 16 * U) * (12 + o.entropy[w]))
    st = f64(stats).reshape(rows, 2)
    close(st[w, 1], o.logsum[w], tol)
    at = ids[:rows * top].cpu().numpy().reshape(rows, top).astype(np.int64)
    best = np.take_along_axis(o.logp, at, 1)
    size = np.where(np.isfinite(best), np.abs(best), 0.0)
    close(f64(tlp[:rows * top]).reshape(rows, top)[w], best[w], tol[:, None] + 8 * U * size[w])

    gen = torch.Generator().manual_seed(3)
    a, b = torch.randn(rows, generator=gen), torch.randn(rows, generator=gen)
    g = torch.empty(rows * vocab, dtype=dt, device=DEV)
    B.dct_lm_logprobs_bwd(flat, rows, vocab, vocab, inv_t, tokens.to(DEV), stats, ent, a.to(DEV), b.to(DEV), g, vocab)
    m = np.where(w, 0.0, st[:, 0])
    want = lm.log_probs_bwd(xs, inv, tokens.numpy(), m, st[:, 1], f64(ent), f64(a), f64(b))
    with np.errstate(invalid="ignore"):
        lpx = np.maximum(xs * inv - m[:, None] - st[:, 1:], -1e4)
    p = np.exp(lpx)
    rel = U * (32 + 8 * np.abs(lpx) + 4 * (np.abs(m) + np.abs(st[:, 1]))[:, None])
    tol = inv * rel * p * (np.abs(f64(a)) + np.abs(f64(b)))[:, None] * (1 + np.abs(lpx) + f64(ent)[:, None]) + half_step(dt) * np.abs(want) * 1.01
    tol[np.arange(rows), tokens.numpy()] += inv * 4 * U * np.abs(f64(a))
    close(f64(g).reshape(rows, vocab), want, tol + 1e-37)


def check_distill_of_masked(dtype, fill, inv_t, rows, vocab, top, tail, monkeypatch):
    """check_distill with the oracle given the far rows from their largest value on: the same distributions, with tolerances that
    do not grow with the mask."""
    dt = DT[dtype]
    x, _ = masked_rows(rows, vocab, torch.finfo(dt).min if fill == "lowest" else fill, dt, vocab + 5)
    gen = torch.Generator().manual_seed(13)
    ids = torch.stack([torch.randperm(vocab - 2, generator=gen)[:top] for _ in range(rows)]).to(torch.int32) + 1
    ids[torch.arange(rows) % 7 == 5] = ids[torch.arange(rows) % 7 == 5] // 3 * 3      # (named twice or more, some of them)
    t = torch.log_softmax(2.0 * torch.randn(rows, top, generator=gen), 1) - 0.25
    distill, log_probs = lm.distill, lm.log_probs
    monkeypatch.setattr(lm, "distill", lambda z, *rest: distill(from_their_largest(z), *rest))
    monkeypatch.setattr(lm, "log_probs", lambda z, *rest: log_probs(from_their_largest(z), *rest))
    # (a teacher whose whole mass lies on columns at fp32's lowest value: the exact loss is fp32's largest number, and a sum that is
    # within its tolerance may round to infinity)
    most = float(np.finfo(np.float32).max)
    monkeypatch.setattr(base, "close", lambda got, want, tol: close(np.where(np.isposinf(got) & np.isfinite(want) & (want + tol >= most), most, got), want, tol))
    check_distill(x, inv_t, ids, t, tail, torch.rand(rows, generator=gen) + 0.5, vocab, 0, dt)


@pytest.mark.parametrize("rows,vocab,top", FAR_SHAPES)
@pytest.mark.parametrize("inv_t", [1.0, 0.5, 0.6])
@pytest.mark.parametrize("fill", FILLS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tail", [False, True])
def test_distill_of_finite_masks(dtype, fill, inv_t, rows, vocab, top, tail, monkeypatch):
    check_distill_of_masked(dtype, fill, inv_t, rows, vocab, top, tail, monkeypatch)


@pytest.mark.parametrize("fill", FILLS)
@pytest.mark.parametrize("tail", [False, True])
def test_distill_of_finite_masks_in_rows_loaded_twice(fill, tail, monkeypatch):
    check_distill_of_masked("bf16", fill, 0.6, 230, 32768, 1024, tail, monkeypatch)


@pytest.mark.parametrize("rows,d,ld,offset", [(3, 7236, 7236, 0), (3, 7237, 7237, 0), (5, 7500, 7500, 0), (310, 7680, 7680, 0), (4, 7680, 7681, 0),
                                              (310, 8000, 8000, 0), (4, 8191, 8191, 0), (4, 8192, 8197, 0), (4, 8192, 8192, 1),
                                              (3, 4097, 4097, 0), (3, 5000, 5001, 1)])
@pytest.mark.parametrize("dtype,pdtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
def test_layer_norm_of_wide_rows_in_a_ring(rows, d, ld, offset, dtype, pdtype):
    """Widths at which the slots of a CTA come near what it may have of shared memory."""
    base.test_layer_norm(rows, d, ld, offset, dtype, pdtype)


ORDER = """
import sys, torch
from paper_2010_08899_b200 import binding as B

def step(rows, vocab, top, times):
    x = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    ids = torch.arange(rows * top, dtype=torch.int32, device="cuda") % vocab
    t, loss, g = torch.zeros(rows * top, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(x)
    ends = [torch.cuda.Event(enable_timing=True) for _ in range(times + 1)]
    for e in ends:
        e.record()
        B.dct_lm_distill(x, rows, vocab, vocab, 1.0, ids, t, top, B.DCT_DISTILL_RENORM, None, loss, g, vocab)
    torch.cuda.synchronize()
    took = sorted(a.elapsed_time(b) for a, b in zip(ends[2:], ends[3:]))
    return took[len(took) // 2]

if sys.argv[1] == "after":
    step(256, 524288, 64, 3)           # the same kernel with eight CTAs to a row
print(step(4096, 32768, 1024, 12))
"""


def test_time_of_a_call_does_not_depend_on_the_calls_before():
    """A persistent grid of one CTA to a row is as large after a call whose rows were split as in a new process (a grid of the other
    shape's size takes several times as long)."""
    took = [float(subprocess.run([sys.executable, "-c", ORDER, word], cwd=ROOT, capture_output=True, text=True, check=True, timeout=300).stdout)
            for word in ("before", "after")]
    assert took[1] < 1.5 * took[0]


@pytest.fixture
def waits_run_out():
    """Every bounded wait gives up before its first poll.  (The kernels then wait again, with a limit of their own, before they go on.)"""
    B.dct_debug_configure(spin_limit=0)
    yield
    B.dct_debug_configure()


@pytest.mark.parametrize("rows,d,ld", [(1500, 256, 256), (700, 512, 512), (701, 509, 509), (301, 1000, 1000), (1200, 1024, 1024), (601, 4096, 4096),
                                       (600, 4095, 4095), (450, 8192, 8192), (450, 8000, 8001)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layer_norm_whose_waits_run_out(dtype, rows, d, ld, waits_run_out):
    """A wait for a row that gave up leaves no finite number: not in the row, not in its statistics, not in the parameters' gradients."""
    dt = DT[dtype]
    x = torch.randn(rows, ld, device=DEV).to(dt)
    y, mean, rstd = torch.zeros(rows, ld, dtype=dt, device=DEV), vec(rows), vec(rows)
    B.dct_layer_norm_fwd(x, rows, d, ld, None, None, 1e-5, y, ld, mean, rstd)
    assert bool(y[:, :d].isnan().all()) and bool((y[:, d:] == 0).all())
    assert bool(mean[:rows].isnan().all()) and bool(rstd[:rows].isnan().all())
    ones, zeros = torch.ones(rows, device=DEV), torch.zeros(rows, device=DEV)
    dx, dw, db = torch.zeros(rows, ld, dtype=dt, device=DEV), vec(d), vec(d)
    ws = B.new_workspace(B.dct_layer_norm_bwd_workspace_bytes(rows, d))
    B.dct_layer_norm_bwd(x, ld, x, rows, d, ld, None, zeros, ones, dx, ld, dw, db, ws)
    assert bool(dx[:, :d].isnan().all()) and bool((dx[:, d:] == 0).all())
    assert bool(dw[:d].isnan().all()) and bool(db[:d].isnan().all())
    # and nothing of it is left behind
    B.dct_debug_configure()
    B.dct_layer_norm_fwd(x, rows, d, ld, None, None, 1e-5, y, ld, mean, rstd)
    B.dct_layer_norm_bwd(x, ld, x, rows, d, ld, None, zeros, ones, dx, ld, dw, db, ws)
    for t in (y, mean[:rows], rstd[:rows], dx, dw[:d], db[:d]):
        assert bool(t.isfinite().all())


@pytest.mark.parametrize("rows,vocab,top", [(700, 1500, 4), (700, 4000, 4), (500, 16000, 4), (500, 32768, 4), (40, 60000, 4), (230, 32768, 1024), (3, 400000, 16)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tail", [False, True])
def test_distill_whose_waits_run_out(dtype, rows, vocab, top, tail, waits_run_out):
    dt = DT[dtype]
    x = torch.randn(rows, vocab, device=DEV).to(dt)
    ids = (torch.arange(rows * top, device=DEV) % vocab).to(torch.int32)
    t = torch.full((rows * top,), -np.log(2.0 * top), device=DEV)
    loss, g, res = vec(rows), torch.zeros_like(x), B.new_result()
    mode = B.DCT_DISTILL_TAIL if tail else B.DCT_DISTILL_RENORM
    B.dct_lm_distill(x, rows, vocab, vocab, 1.0, ids, t, top, mode, None, loss, g, vocab, res)
    assert B.read_result(res).status == B.DCT_ERR_TIMEOUT
    assert bool(loss[:rows].isnan().all()) and bool(g.isnan().all())
    B.dct_lm_distill(x, rows, vocab, vocab, 1.0, ids, t, top, mode, None, loss, None, 0, res)
    assert B.read_result(res).status == B.DCT_ERR_TIMEOUT and bool(loss[:rows].isnan().all())
    B.dct_debug_configure()
    B.dct_lm_distill(x, rows, vocab, vocab, 1.0, ids, t, top, mode, None, loss, g, vocab, res)
    assert B.read_result(res).status == B.DCT_OK
    assert bool(loss[:rows].isfinite().all()) and bool(g.isfinite().all())


@pytest.mark.parametrize("rows,vocab", [(1, 131072), (90, 131072), (150, 65536)])
def test_logprobs_whose_waits_run_out(rows, vocab, waits_run_out):
    """Rows that are split over CTAs, which wait for one another's sums and columns."""
    x = torch.randn(rows, vocab, device=DEV)
    tok = torch.zeros(rows, dtype=torch.int32, device=DEV)
    lp, ent, stats, ids, tlp, res = vec(rows), vec(rows), vec(2 * rows), vec(5 * rows, torch.int32), vec(5 * rows), B.new_result()
    call = lambda: B.dct_lm_logprobs_fwd(x, rows, vocab, vocab, 1.0, tok, 5, lp, ent, stats, ids, tlp, res)
    call()
    assert B.read_result(res).status == B.DCT_ERR_TIMEOUT
    for t in (lp[:rows], ent[:rows], tlp[:5 * rows]):
        assert bool(t.isnan().all())
    B.dct_debug_configure()
    call()
    assert B.read_result(res).status == B.DCT_OK
    want = torch.log_softmax(x.double(), 1)
    assert torch.allclose(lp[:rows].double(), want[:, 0], atol=1e-4) and torch.equal(ids[:5 * rows].view(rows, 5).long(), want.topk(5, 1).indices)


@pytest.mark.parametrize("dtype,rows,vocab,top", [("f32", 300, 1000, 16), ("bf16", 40, 32768, 64), ("f32", 5, 50021, 40)])
@pytest.mark.parametrize("offset", [0.0, -300.0, 8192.0, 65536.0])
def test_distill_from_teacher_values_with_an_offset(dtype, rows, vocab, top, offset):
    """A common offset of a row's teacher values (logits instead of log-probabilities) changes nothing, and costs no accuracy where
    fp32 holds the values: multiples of 2^-6 here."""
    x, _ = logits(rows, vocab, 91, DT[dtype])
    gen = torch.Generator().manual_seed(17)
    ids = torch.stack([torch.randperm(vocab, generator=gen)[:top] for _ in range(rows)]).to(torch.int32)
    ids[0, 1] = ids[0, 0]
    t = (torch.randn(rows, top, generator=gen) * 128).round() / 64 + offset
    check_distill(x, 1.0, ids, t, False, None, vocab, 0, DT[dtype])


def test_a_step_keeps_what_each_of_its_calls_reports():
    """A teacher's column outside the vocabulary is in the step's status when the step is over."""
    from paper_2010_08899_b200.student import Student
    s = Student(64, 301, 8, keep=64, top=4, density=1.0, dtype=torch.float32)
    teach = s.teach

    def teach_badly(teacher):
        teach(teacher)
        s.ids[3] = 301

    s.teach = teach_badly
    r = s.step(torch.randn(8, 64, device=DEV), torch.randn(8, 301, device=DEV))
    assert B.read_result(s.status).status == B.DCT_ERR_BAD_MASK
    assert B.read_result(r.sent).status == B.DCT_OK and B.read_result(s.applied).status == B.DCT_OK
