"""Further edges of the layer norm and of the calls on rows of logits: masks, widths and shapes at which a choice of
kernel or of arithmetic changes.  Tolerances as in test_gpu_lm.py."""
import numpy as np
import pytest
import torch

from oracle import lm
from paper_2010_08899_b200 import binding as B

from .test_gpu_lm import DEV, DT, U, chain, close, f64, half_step, teacher_of, vec

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
