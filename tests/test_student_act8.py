"""The feed-forward block in 8 bits and the student that has one: forward and backward against the same steps in 64 bits, with the same
roundings into 8 bits at the same places."""
import numpy as np
import pytest
import torch

from oracle import act8 as o
from oracle import lm
from paper_2010_08899_b200 import binding as B
from paper_2010_08899_b200 import inputs

pytestmark = pytest.mark.gpu

DEV = "cuda"


def f64(t):
    return t.detach().double().cpu().numpy()


def held(x):
    return o.values(o.hold(x))


def near(got, want, far=2.0 ** -7):
    """Roundings at the same places give the same values but where a sum's last digits decide between two codes (or two bf16 numbers on the
    way): a few in a thousand, each off by at most a sixteenth to an eighth.  A mistake in any factor is off by far more than 2^-7 of the whole."""
    want = np.asarray(want)
    return np.linalg.norm(f64(got).reshape(want.shape) - want) <= far * np.linalg.norm(want)


def block_forward(x, gate, up, down, gelu=False):
    x8 = held(x)
    g, u = x8 @ held(gate).T, x8 @ held(up).T
    h8 = held(o.activation(g, gelu)[0] * u)
    return h8 @ held(down).T, x8, held(g), held(u)


def block_backward(dy, gate, up, down, x8, g, u, as_dtype, gelu=False):
    dh = as_dtype(held(dy) @ held(down.T).T)
    act, slope = o.activation(g, gelu)
    dg, du, h = dh * u * slope, dh * act, act * u
    x8_t, dy8_t = held(x8.T), held(dy.T)
    return (held(dg) @ held(gate.T).T + held(du) @ held(up.T).T, held(dg.T) @ x8_t.T, held(du.T) @ x8_t.T, dy8_t @ held(h.T).T)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,d,f,gelu", [(1, 64, 128, False), (40, 200, 300, True), (130, 256, 520, False), (300, 96, 130, True)])
def test_feed_forward_block(rows, d, f, gelu, dtype):
    from paper_2010_08899_b200.student import FeedForward
    g = torch.Generator(device=DEV).manual_seed(rows)
    params, grads = torch.randn(3 * f * d, generator=g, device=DEV) * d ** -0.5, torch.full((3 * f * d,), 9.0, device=DEV)
    block = FeedForward(d, f, rows, params, grads, B.DCT_ACT_GELU if gelu else B.DCT_ACT_SILU, dtype=dtype)
    block.load()
    x = torch.randn(rows, d, generator=g, device=DEV).to(dtype)
    dy = (torch.randn(rows, d, generator=g, device=DEV) / rows).to(dtype)
    y = block.forward(x).clone()
    dx = block.backward(dy)
    w = [f64(p) for p in (block.gate, block.up, block.down)]
    want, x8, kg, ku = block_forward(f64(x), *w, gelu)
    assert near(y, want)
    as_dtype = (lambda v: v) if dtype == torch.float32 else (lambda v: torch.from_numpy(v).to(dtype).double().numpy())
    back = block_backward(f64(dy), *w, x8, kg, ku, as_dtype, gelu)
    for got, expected in zip((dx, block.grad_gate, block.grad_up, block.grad_down), back):
        assert near(got, expected)
    # serving keeps nothing and gives the same
    before = block.kept_gate.codes.clone()
    assert torch.equal(block.forward(x, keep=False), y) and torch.equal(block.kept_gate.codes, before)


def test_the_blocks_gradients_are_the_formulas():
    """Against the block without any rounding: each of a product's factors is off by at most 2^-4 of an element, 2^-4 / sqrt 3 on average over a
    uniform error, and no more than four such roundings follow one another: 4 * 2^-4 / sqrt 3 = 0.145 of the whole."""
    from paper_2010_08899_b200.student import FeedForward
    rows, d, f = 256, 384, 512
    g = torch.Generator(device=DEV).manual_seed(5)
    params, grads = torch.randn(3 * f * d, generator=g, device=DEV) * d ** -0.5, torch.zeros(3 * f * d, device=DEV)
    block = FeedForward(d, f, rows, params, grads)
    block.load()
    x, dy = torch.randn(rows, d, generator=g, device=DEV).bfloat16(), torch.randn(rows, d, generator=g, device=DEV).bfloat16()
    y = block.forward(x).clone()
    dx = block.backward(dy)
    vx, w = x.double().requires_grad_(), [p.double().detach().requires_grad_() for p in (block.gate, block.up, block.down)]
    out = (torch.nn.functional.silu(vx @ w[0].T) * (vx @ w[1].T)) @ w[2].T
    out.backward(dy.double())
    for got, want in ((y, out.detach()), (dx, vx.grad), (block.grad_gate, w[0].grad), (block.grad_up, w[1].grad), (block.grad_down, w[2].grad)):
        assert float((got.double() - want).norm() / want.norm()) < 0.145


@pytest.mark.parametrize("ffn", [0, 160])
def test_one_step_of_a_student_in_8_bits(ffn):
    """fp32 activations, every activation kept, every gradient sent: the whole step in numpy, rounded into 8 bits at the same places."""
    from paper_2010_08899_b200.student import Student
    rows, d, vocab, top = 24, 96, 701, 12
    s = Student(d, vocab, rows, keep=d, top=top, density=1.0, tail=False, lr=0.25, dtype=torch.float32, seed=3, ffn=ffn, eight_bit=True)
    hidden, teacher = inputs.mp_gradients(rows, d, 1, device=DEV), inputs.lm_logits(rows, vocab, 2, device=DEV)
    before = f64(s.params)
    r = s.step(hidden, teacher)
    head = 2 * d + vocab * d
    w, b, proj = before[:d], before[d:2 * d], before[2 * d:head].reshape(vocab, d)
    weights = [p.reshape(q) for p, q in zip(np.split(before[head:], 3), ((ffn, d), (ffn, d), (d, ffn)))] if ffn else None
    x, t = f64(hidden), f64(teacher)
    z0 = x
    if ffn:
        added, *kept = block_forward(x, *weights)
        z0 = x + added
    n = lm.layer_norm_fwd(z0, w, b, float(np.float32(1e-5)))
    z = held(n.y) @ held(proj).T
    logp = lm.log_probs(t, 1.0).logp
    ids = np.stack([lm.top_columns(t[i], top) for i in range(rows)])
    dist = lm.distill(z, 1.0, ids, np.take_along_axis(logp, ids.astype(np.int64), 1), False, np.full(rows, 1.0 / rows))
    dproj, dy = held(dist.grad.T) @ held(held(n.y).T).T, held(dist.grad) @ held(proj.T).T
    back = lm.layer_norm_bwd(dy, z0, w, n.mean, n.rstd)
    grads, dx = [back.dweight, back.dbias, dproj.reshape(-1)], back.dx
    if ffn:
        added, *weight_grads = block_backward(back.dx, *weights, *kept, lambda v: v)
        dx = dx + added
        grads += [v.reshape(-1) for v in weight_grads]
    assert near(r.loss, dist.loss) and near(r.grad_hidden, dx, 2.0 ** -5)
    got = np.split(f64(s.grads), np.cumsum([v.size for v in grads])[:-1])
    for have, want in zip(got, grads):
        assert np.linalg.norm(have - want) <= 2.0 ** -5 * np.linalg.norm(want)
    assert np.allclose(f64(s.params), before - 0.25 * f64(s.grads), rtol=0, atol=1e-6)
    assert B.read_result(r.sent).count == s.params.numel()
    lp, ent, tops, lps = s.score(hidden, torch.from_numpy(ids[:, 0].astype(np.int32)).to(DEV), alternatives=3)
    assert bool(torch.isfinite(lp).all()) and int(tops.max()) < vocab


def test_the_block_captured_forward_and_backward():
    from paper_2010_08899_b200.student import FeedForward
    rows, d, f = 70, 128, 256
    g = torch.Generator(device=DEV).manual_seed(9)
    params, grads = torch.randn(3 * f * d, generator=g, device=DEV) * d ** -0.5, torch.zeros(3 * f * d, device=DEV)
    block = FeedForward(d, f, rows, params, grads)
    x, dy = torch.randn(rows, d, generator=g, device=DEV).bfloat16(), torch.randn(rows, d, generator=g, device=DEV).bfloat16()
    block.load()
    want = [block.forward(x).clone(), block.backward(dy).clone(), grads.clone()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block.load()
        y = block.forward(x)
        dx = block.backward(dy)
    for _ in range(2):
        grads.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(dx, want[1]) and torch.equal(grads, want[2])
    x.mul_(2.0)                             # new inputs in the same place
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, block.forward(x))


def student_in_8_bits(seed=4):
    from paper_2010_08899_b200.student import Student
    rows, d, vocab, ffn = 24, 96, 701, 160
    s = Student(d, vocab, rows, keep=d, top=12, density=1.0, tail=False, lr=0.25, seed=seed, ffn=ffn, eight_bit=True)
    return s, inputs.mp_gradients(rows, d, 1, device=DEV).bfloat16(), inputs.lm_logits(rows, vocab, 2, device=DEV).bfloat16()


def test_parameters_changed_between_two_calls():
    s, hidden, _ = student_in_8_bits()
    other, _, _ = student_in_8_bits(seed=5)
    s.logits(hidden)
    s.params.copy_(other.params)
    assert torch.equal(s.logits(hidden), other.logits(hidden))
    # serving that changes nothing need not read the parameters again
    assert torch.equal(s.logits(hidden, reload=False), other.logits(hidden))


def test_a_captured_step_trains_the_parameters_it_finds():
    s, hidden, teacher = student_in_8_bits()
    eager, _, _ = student_in_8_bits()
    for _ in range(3):
        eager.step(hidden, teacher)
    start = s.params.clone()
    s.step(hidden, teacher)
    s.params.copy_(start)
    s.residual.zero_()
    s.logits(hidden)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.step(hidden, teacher)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(s.params, eager.params)
    assert torch.equal(s.logits(hidden), eager.logits(hidden))


def test_no_gradients_of_a_pass_that_kept_nothing():
    from paper_2010_08899_b200.student import FeedForward
    rows, d, f = 20, 64, 128
    g = torch.Generator(device=DEV).manual_seed(11)
    params, grads = torch.randn(3 * f * d, generator=g, device=DEV) * d ** -0.5, torch.zeros(3 * f * d, device=DEV)
    block = FeedForward(d, f, rows, params, grads)
    block.load()
    x = torch.randn(rows, d, generator=g, device=DEV).bfloat16()
    with pytest.raises(RuntimeError, match="kept nothing"):
        block.backward(x)
    want = block.forward(x).clone()
    block.backward(x)
    block.forward(x, keep=False)
    with pytest.raises(RuntimeError, match="kept nothing"):
        block.backward(x)
    assert torch.equal(block.forward(x), want)
    block.backward(x)


def test_the_block_refuses_other_shapes_and_parameters_it_never_loaded():
    from paper_2010_08899_b200.student import FeedForward
    rows, d, f = 20, 64, 128
    g = torch.Generator(device=DEV).manual_seed(12)
    params, grads = torch.randn(3 * f * d, generator=g, device=DEV) * d ** -0.5, torch.zeros(3 * f * d, device=DEV)
    block = FeedForward(d, f, rows, params, grads)
    x = torch.randn(rows, d, generator=g, device=DEV).bfloat16()
    with pytest.raises(RuntimeError, match="load"):
        block.forward(x)
    block.load()
    want = [block.forward(x).clone(), block.backward(x).clone()]
    for shape in ((rows, 2 * d), (2 * rows, d), (d, rows), (1, rows, d)):
        other = torch.zeros(shape, device=DEV, dtype=torch.bfloat16)
        with pytest.raises(ValueError, match="x: expected"):
            block.forward(other)
        with pytest.raises(ValueError, match="dy: expected"):
            block.backward(other)
    assert torch.equal(block.forward(x), want[0]) and torch.equal(block.backward(x), want[1])
