"""Measured cases of the operators around a language model's split and at its end: layer norm forward and
backward, log-probabilities of given tokens with entropy and top alternatives (forward and backward), and
distillation from a teacher's top log-probabilities (loss and gradient in one call).

``own`` chooses what ``run`` does: the operators written out in elementary torch operations in 32 bits, or the
calls of :mod:`paper_2010_08899_b200.binding`.  ``exact`` gives the same results from the definitions in 64 bits.
"""
import math

import torch

own = False

KINDS = ("norm_fwd", "norm_bwd", "logp_fwd", "logp_bwd", "distill")
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


def listed():
    return [
        # the norm of one decoding step: a few sequences, one token each; latency alone counts
        {"name": "norm_fwd_decode", "kind": "norm_fwd", "rows": 8, "d": 4096, "pad": 0, "dtype": "bf16", "params": "bf16"},
        # a training batch at the width whose activations the row top-k packs
        {"name": "norm_fwd_train", "kind": "norm_fwd", "rows": 16384, "d": 4096, "pad": 0, "dtype": "bf16", "params": "bf16"},
        # the Transformer width 512 in fp32, a batch that is no multiple of anything
        {"name": "norm_bwd_512_f32", "kind": "norm_bwd", "rows": 4001, "d": 512, "pad": 0, "dtype": "f32", "params": "f32"},
        # the training batch again, with fp32 master parameters
        {"name": "norm_bwd_train", "kind": "norm_bwd", "rows": 16384, "d": 4096, "pad": 0, "dtype": "bf16", "params": "f32"},
        # an odd width: no row but the first starts on a 16-byte boundary
        {"name": "norm_bwd_odd", "kind": "norm_bwd", "rows": 2047, "d": 5003, "pad": 0, "dtype": "bf16", "params": "bf16"},
        # one decoding step of one sequence: the sampled token's log-probability and twenty alternatives
        {"name": "logp_one_token", "kind": "logp_fwd", "rows": 1, "vocab": 131072, "pad": 0, "dtype": "bf16", "top": 20,
         "inv_t": 1.0, "masked": False},
        # constrained decoding of a small batch: most columns masked, some rows down to a few allowed tokens
        {"name": "logp_batch_masked", "kind": "logp_fwd", "rows": 37, "vocab": 50021, "pad": 0, "dtype": "f32", "top": 5,
         "inv_t": 1.25, "masked": True},
        # a teacher's pass over a batch: the message to the student is the best 64 of every row
        {"name": "logp_teacher", "kind": "logp_fwd", "rows": 4096, "vocab": 32768, "pad": 0, "dtype": "bf16", "top": 64,
         "inv_t": 1.0, "masked": False},
        # policy gradient with an entropy bonus: gradient of log-probability and entropy, fp32, padded rows
        {"name": "logp_bwd_policy", "kind": "logp_bwd", "rows": 1023, "vocab": 50021, "pad": 27, "dtype": "f32",
         "inv_t": 1.0, "masked": False},
        # a small student batch at the vocabulary of a small translation model
        {"name": "distill_small", "kind": "distill", "rows": 64, "vocab": 10007, "pad": 0, "dtype": "f32", "top": 16,
         "inv_t": 0.5, "tail": False},
        # the student's step on the teacher's message above
        {"name": "distill_train", "kind": "distill", "rows": 4096, "vocab": 32768, "pad": 0, "dtype": "bf16", "top": 64,
         "inv_t": 1.0, "tail": False},
        # a large vocabulary, the teacher's remaining mass as one more class
        {"name": "distill_wide_tail", "kind": "distill", "rows": 1024, "vocab": 131072, "pad": 0, "dtype": "bf16", "top": 128,
         "inv_t": 1.0, "tail": True},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(KINDS)
    dtype = rng.choice(("bf16", "f32"))
    es = 2 if dtype == "bf16" else 4
    if kind.startswith("norm"):
        d = _log_uniform(rng, 64, 8192)
        if rng.random() < 0.5:
            d = (d + 63) // 64 * 64
        rows = _log_uniform(rng, 1, max(2, min(65536, (1 << 27) // (d * es))))
        return {"kind": kind, "rows": rows, "d": d, "pad": rng.choice((0, 0, 8, 5)), "dtype": dtype,
                "params": rng.choice((dtype, "f32"))}
    vocab = _log_uniform(rng, 1000, 262144)
    if rng.random() < 0.5:
        vocab = (vocab + 63) // 64 * 64
    rows = _log_uniform(rng, 1, max(2, min(16384, (1 << 28) // (vocab * es))))
    case = {"kind": kind, "rows": rows, "vocab": vocab, "pad": rng.choice((0, 0, 16, 3)), "dtype": dtype,
            "inv_t": rng.choice((1.0, 0.5, 1.25))}
    if kind == "logp_fwd":
        case.update(top=_log_uniform(rng, 1, 128), masked=rng.random() < 0.25)
    elif kind == "logp_bwd":
        case.update(masked=rng.random() < 0.25)
    else:
        case.update(top=_log_uniform(rng, 1, 256), tail=rng.random() < 0.5)
    return case


# --------------------------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------------------------

def _logits(rows, vocab, ld, dtype, gen, masked):
    """Logits as a language model gives them: a unigram slope over the columns, noise, and in two rows of three one
    favoured column.  Returns them with the favoured columns.  With ``masked`` nine columns of ten are -inf, in every
    eighth row all but three.  Columns beyond the vocabulary hold a large value that no result may show."""
    dev = "cuda"
    x = torch.full((rows, ld), 1.0e4, device=dev, dtype=dtype)
    rank = torch.randperm(vocab, generator=gen, device=dev).float() + 1.0
    slope = -0.7 * torch.log(rank)
    target = torch.randint(0, vocab, (rows,), generator=gen, device=dev)
    lift = torch.where(torch.rand(rows, generator=gen, device=dev) < 0.67,
                       4.0 + 8.0 * torch.rand(rows, generator=gen, device=dev), torch.zeros((), device=dev))
    step = max(1, (1 << 26) // vocab)
    for lo in range(0, rows, step):
        hi = min(rows, lo + step)
        z = torch.randn(hi - lo, vocab, generator=gen, device=dev) * 2.0 + slope
        z.scatter_add_(1, target[lo:hi, None], lift[lo:hi, None])
        if masked:
            few = (torch.arange(lo, hi, device=dev) % 8 == 7)[:, None]
            keep = torch.rand(hi - lo, vocab, generator=gen, device=dev) < 0.1
            first = torch.arange(vocab, device=dev)[None, :]
            allowed = torch.randint(0, vocab, (hi - lo, 3), generator=gen, device=dev)
            three = (first == allowed[:, :1]) | (first == allowed[:, 1:2]) | (first == allowed[:, 2:])
            keep = torch.where(few, three, keep)
            keep.scatter_(1, target[lo:hi, None], True)
            z = torch.where(keep, z, torch.full((), -math.inf, device=dev))
        x[lo:hi, :vocab] = z.to(dtype)
    return x, target


def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    dt = DTYPES[case["dtype"]]
    rows = case["rows"]
    s = {"case": case}
    if case["kind"].startswith("norm"):
        d, pdt = case["d"], DTYPES[case["params"]]
        ld = d + case["pad"]
        scale = torch.exp(0.5 * torch.randn(rows, 1, generator=gen, device=dev))
        x = (torch.randn(rows, ld, generator=gen, device=dev) * scale + 0.3).to(dt)
        s.update(x=x, ld=ld,
                 weight=(1.0 + 0.2 * torch.randn(d, generator=gen, device=dev)).to(pdt),
                 bias=(0.1 * torch.randn(d, generator=gen, device=dev)).to(pdt),
                 mean=torch.empty(rows, device=dev), rstd=torch.empty(rows, device=dev))
        if case["kind"] == "norm_fwd":
            s["y"] = torch.empty(rows, d, device=dev, dtype=dt)
            return s
        v = x[:, :d].float()
        s["mean"] = v.mean(1)
        s["rstd"] = 1.0 / torch.sqrt(((v - s["mean"][:, None]) ** 2).mean(1) + EPS)
        s["dy"] = torch.randn(rows, d, generator=gen, device=dev).to(dt)
        s["dx"] = torch.empty(rows, d, device=dev, dtype=dt)
        s["dweight"] = torch.empty(d, device=dev)
        s["dbias"] = torch.empty(d, device=dev)
        # enough for any implementation's partial sums of the parameter gradients
        s["workspace"] = torch.empty(2 * 4 * 1024 * (d + 64), device=dev, dtype=torch.uint8)
        return s

    vocab, ld = case["vocab"], case["vocab"] + case["pad"]
    x, target = _logits(rows, vocab, ld, dt, gen, case.get("masked", False))
    s.update(logits=x, ld=ld)
    if case["kind"] != "distill":
        tokens = torch.where(torch.rand(rows, generator=gen, device=dev) < 0.7, target,
                             torch.randint(0, vocab, (rows,), generator=gen, device=dev))
        if rows > 1:       # a prompt's or padding's position: no token is asked for
            tokens = torch.where(torch.rand(rows, generator=gen, device=dev) < 0.05, torch.full_like(tokens, -1), tokens)
        s["tokens"] = tokens.to(torch.int32)
    if case["kind"] == "logp_fwd":
        k = case["top"]
        s.update(logprob=torch.empty(rows, device=dev), entropy=torch.empty(rows, device=dev),
                 stats=torch.empty(rows, 2, device=dev), top_ids=torch.empty(rows, k, device=dev, dtype=torch.int32),
                 top_logprobs=torch.empty(rows, k, device=dev))
    elif case["kind"] == "logp_bwd":
        z = _scaled(x, vocab, case["inv_t"])
        m, logsum, ent = _row_stats(z)
        s.update(stats=torch.stack((m, logsum), 1), entropy=ent,
                 grad_logprob=torch.randn(rows, generator=gen, device=dev),
                 grad_entropy=0.1 * torch.randn(rows, generator=gen, device=dev),
                 grad_logits=torch.empty(rows, ld, device=dev, dtype=dt))
    else:
        k = min(case["top"], vocab)
        ids = torch.empty(rows, k, device=dev, dtype=torch.int32)
        lps = torch.empty(rows, k, device=dev)
        step = max(1, (1 << 26) // vocab)
        for lo in range(0, rows, step):       # a teacher that agrees with the student in the main
            z = x[lo:lo + step, :vocab].float() * case["inv_t"]
            z = z + 0.7 * torch.randn(z.shape, generator=gen, device=dev)
            v, i = torch.topk(z, k, dim=1)
            ids[lo:lo + step] = i.to(torch.int32)
            lps[lo:lo + step] = v - torch.logsumexp(z, 1, keepdim=True)
        s.update(teacher_ids=ids, teacher_logprobs=lps,
                 grad_loss=torch.where(torch.rand(rows, generator=gen, device=dev) < 0.05, 0.0, 1.0) / rows,
                 loss=torch.empty(rows, device=dev), grad_logits=torch.empty(rows, ld, device=dev, dtype=dt))
    return s


# --------------------------------------------------------------------------------------------------------------
# the operators in elementary operations, 32 bits
# --------------------------------------------------------------------------------------------------------------

def _scaled(x, vocab, inv_t):
    z = x[:, :vocab].float()
    return z if inv_t == 1.0 else z * inv_t


def _row_stats(z):
    m = z.amax(1)
    t = z - m[:, None]
    e = torch.exp(t)
    total = e.sum(1)
    logsum = torch.log(total)
    return m, logsum, logsum - torch.where(e > 0, e * t, 0.0).sum(1) / total


def _plain_norm_fwd(s):
    c = s["case"]
    x = s["x"][:, :c["d"]].float()
    mean = x.mean(1)
    xc = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((xc * xc).mean(1) + EPS)
    y = xc * rstd[:, None] * s["weight"].float() + s["bias"].float()
    return {"y": y.to(s["x"].dtype), "mean": mean, "rstd": rstd}


def _plain_norm_bwd(s):
    c = s["case"]
    x, dy = s["x"][:, :c["d"]].float(), s["dy"].float()
    h = (x - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * s["weight"].float()
    dx = s["rstd"][:, None] * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    return {"dx": dx.to(s["x"].dtype), "dweight": (dy * h).sum(0), "dbias": dy.sum(0)}


def _top(x, k):
    """The k largest of each row, best first, equal values by the lower column: one whole key per element."""
    bits = (x + 0.0).view(torch.int32).long()
    order = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF) - 1)
    key = order * (1 << 32) + (0xFFFFFFFF - torch.arange(x.shape[1], device=x.device))
    return torch.topk(key, k, dim=1).indices


def _plain_logp_fwd(s):
    c = s["case"]
    x = s["logits"][:, :c["vocab"]].float()
    z = _scaled(x, c["vocab"], c["inv_t"])
    m, logsum, ent = _row_stats(z)
    tok = s["tokens"].long()
    lp = z.gather(1, tok.clamp_min(0)[:, None])[:, 0] - m - logsum
    top = _top(x, c["top"])
    return {"logprob": torch.where(tok >= 0, lp, 0.0), "entropy": ent, "stats": torch.stack((m, logsum), 1),
            "top_ids": top.to(torch.int32), "top_logprobs": z.gather(1, top) - m[:, None] - logsum[:, None]}


def _plain_logp_bwd(s):
    c = s["case"]
    z = _scaled(s["logits"], c["vocab"], c["inv_t"])
    lp = z - s["stats"][:, :1] - s["stats"][:, 1:]
    p = torch.exp(lp)
    tok = s["tokens"].long()
    a = torch.where(tok >= 0, s["grad_logprob"], 0.0)[:, None]
    plogp = torch.where(p > 0, p * (lp + s["entropy"][:, None]), 0.0)
    g = -a * p - s["grad_entropy"][:, None] * plogp
    g.scatter_add_(1, tok.clamp_min(0)[:, None], a)
    return {"grad_logits": (g * c["inv_t"]).to(s["logits"].dtype)}


def _plain_distill(s):
    c = s["case"]
    z = _scaled(s["logits"], c["vocab"], c["inv_t"])
    ids, t = s["teacher_ids"].long(), s["teacher_logprobs"]
    lp = z - z.amax(1, keepdim=True)
    lp = lp - torch.log(torch.exp(lp).sum(1, keepdim=True))
    if c["tail"]:
        q, logq = torch.exp(t), t
        q_r = (1.0 - q.sum(1)).clamp_min(0.0)
        rest = lp.scatter(1, ids, -math.inf)
        rest_max = rest.amax(1, keepdim=True)
        u = torch.exp(rest - rest_max)
        total = u.sum(1, keepdim=True)
        log_p_r = (rest_max + torch.log(total))[:, 0]
        grad = (u / total) * (torch.exp(log_p_r) - q_r)[:, None]
        extra = torch.where(q_r > 0, q_r * (torch.log(q_r) - log_p_r), 0.0)
        grad.scatter_(1, ids, torch.exp(lp.gather(1, ids)) - q)
    else:
        logq = t - t.amax(1, keepdim=True)
        logq = logq - torch.log(torch.exp(logq).sum(1, keepdim=True))
        q, extra = torch.exp(logq), 0.0
        grad = torch.exp(lp)
        grad.scatter_add_(1, ids, -q)
    loss = (q * (logq - lp.gather(1, ids))).sum(1) + extra
    return {"loss": loss, "grad_logits": (grad * (s["grad_loss"] * c["inv_t"])[:, None]).to(s["logits"].dtype)}


# --------------------------------------------------------------------------------------------------------------
# the framework's calls
# --------------------------------------------------------------------------------------------------------------

def _own_run(s):
    from paper_2010_08899_b200 import binding as B
    c = s["case"]
    kind, rows = c["kind"], c["rows"]
    if kind == "norm_fwd":
        B.dct_layer_norm_fwd(s["x"], rows, c["d"], s["ld"], s["weight"], s["bias"], EPS, s["y"], c["d"], s["mean"], s["rstd"])
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    if kind == "norm_bwd":
        B.dct_layer_norm_bwd(s["dy"], c["d"], s["x"], rows, c["d"], s["ld"], s["weight"], s["mean"], s["rstd"],
                             s["dx"], c["d"], s["dweight"], s["dbias"], s["workspace"])
        return {"dx": s["dx"], "dweight": s["dweight"], "dbias": s["dbias"]}
    if kind == "logp_fwd":
        B.dct_lm_logprobs_fwd(s["logits"], rows, c["vocab"], s["ld"], c["inv_t"], s["tokens"], c["top"],
                              s["logprob"], s["entropy"], s["stats"], s["top_ids"], s["top_logprobs"])
        return {k: s[k] for k in ("logprob", "entropy", "stats", "top_ids", "top_logprobs")}
    if kind == "logp_bwd":
        B.dct_lm_logprobs_bwd(s["logits"], rows, c["vocab"], s["ld"], c["inv_t"], s["tokens"], s["stats"], s["entropy"],
                              s["grad_logprob"], s["grad_entropy"], s["grad_logits"], s["ld"])
        return {"grad_logits": s["grad_logits"][:, :c["vocab"]]}
    B.dct_lm_distill(s["logits"], rows, c["vocab"], s["ld"], c["inv_t"], s["teacher_ids"], s["teacher_logprobs"],
                     s["teacher_ids"].shape[1], B.DCT_DISTILL_TAIL if c["tail"] else B.DCT_DISTILL_RENORM,
                     s["grad_loss"], s["loss"], s["grad_logits"], s["ld"])
    return {"loss": s["loss"], "grad_logits": s["grad_logits"][:, :c["vocab"]]}


def run(state):
    if own:
        return _own_run(state)
    return {"norm_fwd": _plain_norm_fwd, "norm_bwd": _plain_norm_bwd, "logp_fwd": _plain_logp_fwd,
            "logp_bwd": _plain_logp_bwd, "distill": _plain_distill}[state["case"]["kind"]](state)


# --------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------------------------------------------

def work(case):
    es, rows = (2 if case["dtype"] == "bf16" else 4), case["rows"]
    if case["kind"].startswith("norm"):
        n, ps = rows * case["d"], (2 if case["params"] == "bf16" else 4)
        if case["kind"] == "norm_fwd":
            return {"bytes": 2 * n * es + 2 * case["d"] * ps + 8 * rows, "flops": 8 * n}
        return {"bytes": 3 * n * es + case["d"] * (ps + 8) + 8 * rows, "flops": 14 * n}
    n = rows * case["vocab"]
    if case["kind"] == "logp_fwd":
        return {"bytes": n * es + rows * (20 + 8 * case["top"]), "flops": 6 * n}
    if case["kind"] == "logp_bwd":
        return {"bytes": 2 * n * es + 24 * rows, "flops": 7 * n}
    return {"bytes": 2 * n * es + rows * (8 + 8 * case["top"]), "flops": 8 * n}


# --------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------------------------------------------

def _exact_norm(case, s):
    d = case["d"]
    x, w, b = s["x"][:, :d].double(), s["weight"].double(), s["bias"].double()
    if case["kind"] == "norm_fwd":
        mean = x.sum(1) / d
        rstd = (((x - mean[:, None]) ** 2).sum(1) / d + EPS) ** -0.5
        return {"y": (x - mean[:, None]) * rstd[:, None] * w + b, "mean": mean, "rstd": rstd}
    dy, r = s["dy"].double(), s["rstd"].double()[:, None]
    h = (x - s["mean"].double()[:, None]) * r
    g = dy * w
    dx = r * (g - g.sum(1, keepdim=True) / d - h * ((g * h).sum(1, keepdim=True) / d))
    return {"dx": dx, "dweight": torch.einsum("ij,ij->j", dy, h), "dbias": dy.sum(0)}


def _exact_rows(case, s, lo, hi):
    """One slice of rows of a vocabulary-wide case."""
    z = s["logits"][lo:hi, :case["vocab"]].double() * case["inv_t"]
    lse = torch.logsumexp(z, 1, keepdim=True)
    lp = z - lse
    p = torch.exp(lp)
    n = torch.arange(hi - lo, device=z.device)
    if case["kind"] == "logp_fwd":
        tok = s["tokens"][lo:hi].long()
        top = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :case["top"]]
        m = z.max(1).values
        return {"logprob": torch.where(tok < 0, 0.0, lp[n, tok.clamp_min(0)]),
                "entropy": torch.special.entr(p).sum(1), "stats": torch.stack((m, lse[:, 0] - m), 1),
                "top_ids": top.to(torch.int32), "top_logprobs": torch.gather(lp, 1, top)}
    if case["kind"] == "logp_bwd":
        tok = s["tokens"][lo:hi].long()
        # from the saved numbers, as the operator is given them
        lp = z - s["stats"][lo:hi].double().sum(1, keepdim=True)
        p = torch.exp(lp)
        a = torch.where(tok < 0, 0.0, s["grad_logprob"][lo:hi].double())
        c = s["grad_entropy"][lo:hi].double()[:, None]
        g = c * (torch.special.entr(p) - p * s["entropy"][lo:hi].double()[:, None]) - a[:, None] * p
        g[n, tok.clamp_min(0)] += a
        return {"grad_logits": g * case["inv_t"]}
    ids, t = s["teacher_ids"][lo:hi].long(), s["teacher_logprobs"][lo:hi].double()
    scale = (s["grad_loss"][lo:hi].double() * case["inv_t"])[:, None]
    if not case["tail"]:
        q = torch.softmax(t, 1)
        loss = (torch.xlogy(q, q) - q * lp.gather(1, ids)).sum(1)
        dense = torch.zeros_like(p).scatter_(1, ids, q)
        return {"loss": loss, "grad_logits": (p - dense) * scale}
    q = torch.exp(t)
    listed_ids = torch.zeros_like(p, dtype=torch.bool).scatter_(1, ids, True)
    q_r = (1.0 - q.sum(1)).clamp_min(0.0)
    p_r = torch.where(listed_ids, 0.0, p).sum(1)
    loss = (torch.xlogy(q, q) - q * lp.gather(1, ids)).sum(1) + torch.xlogy(q_r, q_r / p_r)
    grad = torch.where(listed_ids, p - torch.zeros_like(p).scatter_(1, ids, q), p * (1.0 - q_r / p_r)[:, None])
    return {"loss": loss, "grad_logits": grad * scale}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"].startswith("norm"):
        return _exact_norm(case, s)
    step = max(1, (1 << 25) // case["vocab"])
    parts = [_exact_rows(case, s, lo, min(case["rows"], lo + step)) for lo in range(0, case["rows"], step)]
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
