"""The layer norm, the log-probabilities and the distillation together with the packing: a step of the split student
against the same step in 64 bits, and a few steps of it learning."""
import numpy as np
import pytest
import torch

from oracle import lm
from paper_2010_08899_b200 import binding as B
from paper_2010_08899_b200 import inputs

pytestmark = pytest.mark.gpu

DEV = "cuda"


def f64(t):
    return t.detach().double().cpu().numpy()


@pytest.mark.parametrize("tail", [False, True])
def test_one_step_against_64_bits(tail):
    """fp32 activations, every activation kept, every gradient sent: the whole step restated in numpy.  Each of the few
    products of depth d, rows or vocab loses sqrt(depth) u of its terms' size; a relative 2^-24 * 64 * 16 of the largest
    element is far above that and far below any mistake."""
    from paper_2010_08899_b200.student import Student
    rows, d, vocab, top = 24, 96, 701, 12
    s = Student(d, vocab, rows, keep=d, top=top, density=1.0, tail=tail, temperature=2.0, lr=0.25, dtype=torch.float32, seed=3)
    hidden = inputs.mp_gradients(rows, d, 1, device=DEV)
    teacher = inputs.lm_logits(rows, vocab, 2, device=DEV)
    before = f64(s.params)
    old = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        r = s.step(hidden, teacher)
    finally:
        torch.backends.cuda.matmul.allow_tf32 = old
    w, b, proj = before[:d], before[d:2 * d], before[2 * d:].reshape(vocab, d)
    x, t = f64(hidden), f64(teacher)
    n = lm.layer_norm_fwd(x, w, b, float(np.float32(1e-5)))
    z = n.y @ proj.T
    logp = lm.log_probs(t, 0.5).logp
    ids = np.stack([lm.top_columns(t[i], top) for i in range(rows)])
    o = lm.distill(z, 0.5, ids, np.take_along_axis(logp, ids.astype(np.int64), 1), tail, np.full(rows, 1.0 / rows))
    back = lm.layer_norm_bwd(o.grad @ proj, x, w, n.mean, n.rstd)
    grads = np.concatenate([back.dweight, back.dbias, (o.grad.T @ n.y).reshape(-1)])
    near = lambda got, want: np.abs(f64(got).reshape(want.shape) - want).max() <= 2.0 ** -24 * 64 * 16 * np.abs(want).max()
    assert np.array_equal(s.ids.view(rows, top).cpu().numpy(), ids)
    assert near(r.loss, o.loss) and near(r.grad_hidden, back.dx) and near(s.grads, grads)
    assert near(s.params, before - 0.25 * grads)
    assert B.read_result(r.sent).count == s.params.numel() and not s.residual.any()
    assert B.read_result(s.status).status == B.DCT_OK


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_student_learns_over_the_packed_messages(dtype):
    """A quarter of the activations and a twentieth of the gradients cross; the loss falls all the same, and what is sent
    plus what is kept back is the gradient plus what was kept back before."""
    from paper_2010_08899_b200.student import Student
    rows, d, vocab, top = 128, 256, 5003, 32
    s = Student(d, vocab, rows, keep=d // 4, top=top, density=0.05, dtype=dtype, lr=20.0)
    hidden = inputs.mp_gradients(rows, d, 11, dtype=dtype, device=DEV)
    teacher = inputs.lm_logits(rows, vocab, 12, dtype=dtype, device=DEV)
    tokens = teacher.float().argmax(1).to(torch.int32)
    losses, scores = [], []
    for _ in range(6):
        kept = s.residual.clone()
        r = s.step(hidden, teacher)
        assert torch.equal(s.update + s.residual, s.grads + kept)
        losses.append(float(r.loss.mean()))
        lp, ent, ids, lps = s.score(hidden, tokens, alternatives=4)
        scores.append(float(lp.mean()))
        assert bool((lps[:, 0] >= lp).all()) and bool((ent >= 0).all()) and int(ids.max()) < vocab
    assert losses[-1] < 0.8 * losses[0] and scores[-1] > scores[0]
