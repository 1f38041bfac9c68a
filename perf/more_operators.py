"""Measured cases of a Transformer stage whose activations are held in 8 bits: writing a checkpoint and reading it back,
the matrix product of two such matrices, the weights' gradient from a checkpoint, and the gated feed-forward block forward
and backward.

A matrix in 8 bits is codes in e4m3, ``ld`` bytes to a row, and a power of two for every 128 columns of a row, one byte
``e + 127``: the byte of row r and block b lies at ``((b // 4) * tiles + r // 128) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4``
with ``tiles = ceil(rows / 128)``.  e is the smallest power with which the block's largest magnitude is at most 448 (at least -127).

``own`` chooses what ``run`` does: the operators written out in elementary torch operations in 32 bits, or the
calls of :mod:`paper_2010_08899_b200.binding`.  ``exact`` gives the same results from the definitions in 64 bits.
"""
import math

import torch

own = False

KINDS = ("keep", "product", "weight_grad", "gated_fwd", "gated_bwd")
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
GELU_A, GELU_B = 2.0 * math.sqrt(2.0 / math.pi), 0.044715


def listed():
    return [
        # one decoding step's activations, kept for the next worker: latency alone counts
        {"name": "keep_few", "kind": "keep", "rows": 8, "cols": 4096, "pad": 0, "dtype": "bf16"},
        # a training batch's activations, kept from the forward pass to the backward pass
        {"name": "keep_train", "kind": "keep", "rows": 16384, "cols": 4096, "pad": 0, "dtype": "bf16"},
        # fp32 activations at an odd width inside wider rows: no row but the first starts on a 16-byte boundary
        {"name": "keep_odd_f32", "kind": "keep", "rows": 2047, "cols": 5003, "pad": 6, "dtype": "f32"},
        # a projection in a decoding step of a small batch: the weights' bytes are what counts
        {"name": "product_few", "kind": "product", "m": 16, "n": 8192, "k": 4096, "dtype": "bf16"},
        # sizes that fill no tile, to fp32 logits
        {"name": "product_odd_f32", "kind": "product", "m": 1023, "n": 5003, "k": 2007, "dtype": "f32"},
        # a projection of a training batch
        {"name": "product_train", "kind": "product", "m": 8192, "n": 8192, "k": 4096, "dtype": "bf16"},
        # the gradient of a layer of the Transformer width 512 from a ragged batch: a long sum into a small matrix
        {"name": "weight_grad_512", "kind": "weight_grad", "rows": 4001, "d_out": 512, "d_in": 512, "dtype": "f32"},
        # the gradient of a wide layer over a training batch
        {"name": "weight_grad_train", "kind": "weight_grad", "rows": 16384, "d_out": 8192, "d_in": 4096, "dtype": "f32"},
        # the gated block in a decoding step: dense result, nothing is kept
        {"name": "gated_few", "kind": "gated_fwd", "rows": 4, "d": 4096, "f": 8192, "gelu": False, "kept": False},
        # the gated block of a training batch: result, gate and up stay in 8 bits (and are read back here to be looked at)
        {"name": "gated_train", "kind": "gated_fwd", "rows": 8192, "d": 4096, "f": 8192, "gelu": False, "kept": True},
        # backward of a small block at odd sizes: gradients of the input and of the three weights
        {"name": "gated_bwd_odd", "kind": "gated_bwd", "rows": 777, "d": 1000, "f": 1336, "gelu": True},
        # backward of the training batch
        {"name": "gated_bwd_train", "kind": "gated_bwd", "rows": 8192, "d": 4096, "f": 8192, "gelu": False},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    d = _log_uniform(rng, lo, hi)
    return (d + 63) // 64 * 64 if rng.random() < 0.5 else d


def draw(rng):
    kind = rng.choice(KINDS)
    dtype = rng.choice(("bf16", "f32"))
    if kind == "keep":
        cols = _width(rng, 64, 8192)
        rows = _log_uniform(rng, 1, max(2, min(32768, (1 << 26) // cols)))
        return {"kind": kind, "rows": rows, "cols": cols, "pad": rng.choice((0, 0, 8, 5)), "dtype": dtype}
    if kind == "product":
        n, k = _width(rng, 64, 16384), _width(rng, 64, 8192)
        m = _log_uniform(rng, 1, max(2, min(16384, (1 << 38) // (n * k))))
        return {"kind": kind, "m": m, "n": n, "k": k, "dtype": dtype}
    if kind == "weight_grad":
        d_out, d_in = _width(rng, 64, 8192), _width(rng, 64, 8192)
        rows = _log_uniform(rng, 1, max(2, min(32768, (1 << 38) // (d_out * d_in))))
        return {"kind": kind, "rows": rows, "d_out": d_out, "d_in": d_in, "dtype": dtype}
    d, f = _width(rng, 64, 4096), _width(rng, 64, 8192)
    rows = _log_uniform(rng, 1, max(2, min(16384, (1 << 37) // (d * f))))
    case = {"kind": kind, "rows": rows, "d": d, "f": f, "gelu": rng.random() < 0.5}
    if kind == "gated_fwd":
        case["kept"] = rng.random() < 0.5
    return case


# --------------------------------------------------------------------------------------------------------------
# matrices in 8 bits, 32-bit arithmetic
# --------------------------------------------------------------------------------------------------------------

def _up(n, to):
    return (n + to - 1) // to * to


def _empty8(rows, cols):
    """Buffers of a matrix in 8 bits: (codes [rows, ld], scales, cols)."""
    return (torch.empty(rows, _up(cols, 16), dtype=torch.uint8, device="cuda"),
            torch.empty(_up(rows, 128) * _up(cols, 512) // 128, dtype=torch.uint8, device="cuda"), cols)


def _blocks(x):
    """fp32 [rows, cols] -> codes [rows, blocks, 128], zeros behind the last column, and bytes of the powers [rows, blocks]."""
    rows, cols = x.shape
    v = torch.nn.functional.pad(x, (0, _up(cols, 128) - cols)).view(rows, -1, 128)
    bits = v.abs().amax(2).view(torch.int32)
    byte = (((bits + 0x1FFFFF) >> 23) - 8).clamp(0, 254)
    inverse = ((254 - byte).clamp_min(1) << 23).view(torch.float32)
    return (v * inverse[:, :, None]).to(torch.float8_e4m3fn), byte


def _single(x):
    """fp64 to fp32, but never onto a value of fewer digits that x is next to: such a value may be halfway between two codes."""
    near = x.float()
    return torch.where(near.double() == x, near, torch.nextafter(near, torch.where(x > near, math.inf, -math.inf).float()))


def _quantise(x):
    """The values that 8 bits hold of [rows, cols]."""
    x = _single(x) if x.dtype == torch.float64 else x
    q, byte = _blocks(x)
    return (q.float() * torch.exp2(byte - 127.0)[:, :, None]).view(x.shape[0], -1)[:, :x.shape[1]]


def _encode(x):
    """A matrix in 8 bits (codes, scales, cols) from [rows, cols]."""
    rows, cols = x.shape
    q, byte = _blocks(x.float())
    codes, scales, _ = _empty8(rows, cols)
    codes.fill_(0x55)               # what lies behind the last column is not looked at
    codes[:, :cols] = q.view(torch.uint8).view(rows, -1)[:, :cols]
    whole = torch.full((_up(rows, 128), _up(cols, 512) // 128), 0x5A, dtype=torch.uint8, device=x.device)
    whole[:rows, :byte.shape[1]] = byte.to(torch.uint8)
    r, b = whole.shape
    scales.copy_(whole.view(r // 128, 4, 32, b // 4, 4).permute(3, 0, 2, 1, 4).reshape(-1))
    return codes, scales, cols


def _decode(m):
    """fp32 values of a matrix in 8 bits."""
    codes, scales, cols = m
    rows = codes.shape[0]
    r, b = _up(rows, 128), _up(cols, 512) // 128
    byte = scales.view(b // 4, r // 128, 32, 4, 4).permute(1, 3, 2, 0, 4).reshape(r, b)[:rows, :_up(cols, 128) // 128]
    power = torch.exp2(byte.float() - 127.0)
    return codes[:, :cols].view(torch.float8_e4m3fn).float() * power.repeat_interleave(128, 1)[:, :cols]


# --------------------------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------------------------

def _activations(rows, cols, gen):
    """Rows of different size, a few columns that are far larger than the rest, as a Transformer's activations have them."""
    scale = torch.exp(0.5 * torch.randn(rows, 1, generator=gen, device="cuda"))
    col = torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.01, 20.0, 1.0)
    return torch.randn(rows, cols, generator=gen, device="cuda") * scale * col


def _weights(rows, cols, gen):
    return torch.randn(rows, cols, generator=gen, device="cuda") * cols ** -0.5


def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    kind = case["kind"]
    s = {"case": case}
    if kind == "keep":
        rows, cols, dt = case["rows"], case["cols"], DTYPES[case["dtype"]]
        ld = cols + case["pad"]
        x = torch.full((rows, ld), 1.0e4, device=dev, dtype=dt)
        x[:, :cols] = _activations(rows, cols, gen).to(dt)
        if rows > 2:
            x[rows // 2, :cols] = 0.0                  # a padded position
        s.update(x=x, ld=ld, kept=_empty8(rows, cols), y=torch.empty(rows, cols, device=dev, dtype=dt))
    elif kind == "product":
        m, n, k = case["m"], case["n"], case["k"]
        s.update(a=_encode(_activations(m, k, gen)), b=_encode(_weights(n, k, gen)),
                 c=torch.empty(m, n, device=dev, dtype=DTYPES[case["dtype"]]))
    elif kind == "weight_grad":
        rows, d_out, d_in = case["rows"], case["d_out"], case["d_in"]
        dy = (torch.randn(rows, d_out, generator=gen, device=dev) / rows).to(torch.bfloat16)
        s.update(dy=dy, kept=_encode(_activations(rows, d_in, gen)), dy_t=_empty8(d_out, rows), kept_t=_empty8(d_in, rows),
                 dw=torch.empty(d_out, d_in, device=dev, dtype=DTYPES[case["dtype"]]))
    else:
        rows, d, f = case["rows"], case["d"], case["f"]
        x = _activations(rows, d, gen)
        gate_w, up_w = _weights(f, d, gen), _weights(f, d, gen)
        s["x"] = _encode(x)
        if kind == "gated_fwd":
            s.update(gate_w=_encode(gate_w), up_w=_encode(up_w), h=torch.empty(rows, f, device=dev, dtype=torch.bfloat16))
            if case["kept"]:
                s.update(h8=_empty8(rows, f), gate=_empty8(rows, f), up=_empty8(rows, f),
                         gate_read=torch.empty_like(s["h"]), up_read=torch.empty_like(s["h"]))
        else:
            # the block's own gate and up are of the size that its weights give them
            size = x.square().mean(1, keepdim=True).sqrt()
            s.update(gate=_encode(torch.randn(rows, f, generator=gen, device=dev) * size),
                     up=_encode(torch.randn(rows, f, generator=gen, device=dev) * size),
                     dh=(torch.randn(rows, f, generator=gen, device=dev) / rows).to(torch.bfloat16),
                     dy_t=_encode(torch.randn(d, rows, generator=gen, device=dev) / rows),
                     gate_wt=_encode(gate_w.t().contiguous()), up_wt=_encode(up_w.t().contiguous()),
                     x_t=_empty8(d, rows), dgate=_empty8(rows, f), dup=_empty8(rows, f), dgate_t=_empty8(f, rows),
                     dup_t=_empty8(f, rows), h_t=_empty8(f, rows))
            new = lambda *shape: torch.empty(*shape, device=dev, dtype=torch.bfloat16)
            s.update(dx=new(rows, d), dgate_w=new(f, d), dup_w=new(f, d), ddown_w=new(d, f))
    return s


# --------------------------------------------------------------------------------------------------------------
# the operators in elementary operations, 32 bits
# --------------------------------------------------------------------------------------------------------------

def _share(g, gelu):
    """The activation is g times a share, sigmoid(y): q = sigmoid(-|y|), and the derivative of y."""
    y = GELU_A * (g + GELU_B * g * g * g) if gelu else g
    return torch.sigmoid(-y.abs()), GELU_A * (1.0 + 3.0 * GELU_B * g * g) if gelu else 1.0


def _beside(p, c, up):
    """p + c for a c that is never quite 0: where the sum would be p, the number next to p, away from 0 where ``up``."""
    s = p + c
    return torch.where((s == p) & (p != 0), torch.nextafter(p, torch.where(up, p * math.inf, torch.zeros_like(p))), s)


def _gated(g, u, gelu):
    """act(g) u.  g and u of four digits leave products halfway between two codes, and the share, 1 - q, is just below 1."""
    q, _ = _share(g, gelu)
    p, small = g * u, torch.zeros_like(g, dtype=torch.bool)
    return torch.where(g < 0, g * q * u, _beside(p, -p * q, small))


def _gated_slopes(dh, g, u, gelu):
    """dh u act'(g) and dh act(g), in the same way."""
    q, dy = _share(g, gelu)
    p, small = dh * u, torch.zeros_like(g, dtype=torch.bool)
    more = (g - g * q) * dy - 1.0
    dg = torch.where(g < 0, p * (q + g * q * (1.0 - q) * dy), _beside(p, p * q * more, more > 0))
    return dg, torch.where(g < 0, dh * g * q, _beside(dh * g, -dh * g * q, small))


def _plain_keep(s):
    c = s["case"]
    return {"read": _quantise(s["x"][:, :c["cols"]].float()).to(s["x"].dtype)}


def _plain_product(s):
    return {"c": (_decode(s["a"]) @ _decode(s["b"]).t()).to(s["c"].dtype)}


def _plain_weight_grad(s):
    dy_t = _quantise(s["dy"].float().t().contiguous())
    kept_t = _quantise(_decode(s["kept"]).t().contiguous())
    return {"dw": (dy_t @ kept_t.t()).to(s["dw"].dtype)}


def _plain_gated_fwd(s):
    c = s["case"]
    x = _decode(s["x"])
    g, u = x @ _decode(s["gate_w"]).t(), x @ _decode(s["up_w"]).t()
    h = _gated(g, u, c["gelu"])
    if not c["kept"]:
        return {"h": h.to(torch.bfloat16)}
    return {"h": _quantise(h).to(torch.bfloat16), "gate": _quantise(g).to(torch.bfloat16), "up": _quantise(u).to(torch.bfloat16)}


def _plain_gated_bwd(s):
    g, u, gelu = _decode(s["gate"]).double(), _decode(s["up"]).double(), s["case"]["gelu"]
    dg, du = _gated_slopes(s["dh"].double(), g, u, gelu)
    h = _gated(g, u, gelu)
    dx = _quantise(dg) @ _decode(s["gate_wt"]).t() + _quantise(du) @ _decode(s["up_wt"]).t()
    turned = lambda v: _quantise(v.t().contiguous())
    x_t = turned(_decode(s["x"])).t()
    out = {"dx": dx, "dgate_w": turned(dg) @ x_t, "dup_w": turned(du) @ x_t, "ddown_w": _decode(s["dy_t"]) @ turned(h).t()}
    return {k: v.to(torch.bfloat16) for k, v in out.items()}


# --------------------------------------------------------------------------------------------------------------
# the framework's calls
# --------------------------------------------------------------------------------------------------------------

def _own_run(s):
    from paper_2010_08899_b200 import binding as B
    c = s["case"]
    held = s.get("held")
    if held is None:           # the handles of the buffers, made once as a user's program makes them
        held = s["held"] = {k: B.act8(v[0], v[1], v[0].shape[0], v[2]) for k, v in s.items() if isinstance(v, tuple)}
    if c["kind"] == "keep":
        B.dct_act8_pack(s["x"], c["rows"], c["cols"], s["ld"], held["kept"])
        B.dct_act8_unpack(held["kept"], s["y"], c["cols"])
        return {"read": s["y"]}
    if c["kind"] == "product":
        B.dct_gemm8(held["a"], held["b"], s["c"], c["n"])
        return {"c": s["c"]}
    if c["kind"] == "weight_grad":
        B.dct_act8_pack(s["dy"], c["rows"], c["d_out"], c["d_out"], None, held["dy_t"])
        B.dct_act8_transpose(held["kept"], held["kept_t"])
        B.dct_gemm8(held["dy_t"], held["kept_t"], s["dw"], c["d_in"])
        return {"dw": s["dw"]}
    act = B.DCT_ACT_GELU if c["gelu"] else B.DCT_ACT_SILU
    if c["kind"] == "gated_fwd":
        if not c["kept"]:
            B.dct_gated8_fwd(held["x"], held["gate_w"], held["up_w"], act, None, s["h"], c["f"])
            return {"h": s["h"]}
        B.dct_gated8_fwd(held["x"], held["gate_w"], held["up_w"], act, held["h8"], None, 0, held["gate"], held["up"])
        B.dct_act8_unpack(held["h8"], s["h"], c["f"])
        B.dct_act8_unpack(held["gate"], s["gate_read"], c["f"])
        B.dct_act8_unpack(held["up"], s["up_read"], c["f"])
        return {"h": s["h"], "gate": s["gate_read"], "up": s["up_read"]}
    B.dct_gated8_bwd(s["dh"], c["f"], held["gate"], held["up"], act, held["dgate"], held["dup"], held["dgate_t"], held["dup_t"],
                     held["h_t"])
    B.dct_act8_transpose(held["x"], held["x_t"])
    B.dct_gemm8(held["dgate"], held["gate_wt"], s["dx"], c["d"], held["dup"], held["up_wt"])
    B.dct_gemm8(held["dgate_t"], held["x_t"], s["dgate_w"], c["d"])
    B.dct_gemm8(held["dup_t"], held["x_t"], s["dup_w"], c["d"])
    B.dct_gemm8(held["dy_t"], held["h_t"], s["ddown_w"], c["f"])
    return {k: s[k] for k in ("dx", "dgate_w", "dup_w", "ddown_w")}


def run(state):
    if own:
        return _own_run(state)
    return {"keep": _plain_keep, "product": _plain_product, "weight_grad": _plain_weight_grad, "gated_fwd": _plain_gated_fwd,
            "gated_bwd": _plain_gated_bwd}[state["case"]["kind"]](state)


# --------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------------------------------------------

def _bytes8(rows, cols):
    return rows * cols + rows * (_up(cols, 128) // 128)


def work(case):
    kind = case["kind"]
    es = 4 if case.get("dtype") == "f32" else 2
    if kind == "keep":        # written once and read back
        n = case["rows"] * case["cols"]
        return {"bytes": 2 * n * es + 2 * _bytes8(case["rows"], case["cols"]), "flops": 4 * n}
    if kind == "product":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": _bytes8(m, k) + _bytes8(n, k) + m * n * es, "flops": 2 * m * n * k}
    if kind == "weight_grad":
        r, o, i = case["rows"], case["d_out"], case["d_in"]
        return {"bytes": 2 * r * o + _bytes8(r, i) + o * i * es, "flops": 2 * r * o * i}
    r, d, f = case["rows"], case["d"], case["f"]
    if kind == "gated_fwd":
        # (what is kept is read back)
        return {"bytes": _bytes8(r, d) + 2 * _bytes8(f, d) + (6 * _bytes8(r, f) + 6 * r * f if case["kept"] else 2 * r * f),
                "flops": 4 * r * d * f}
    return {"bytes": _bytes8(r, d) + _bytes8(d, r) + 2 * _bytes8(r, f) + 2 * _bytes8(d, f) + 2 * (r * f + r * d + 3 * f * d),
            "flops": 10 * r * d * f}


# --------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------------------------------------------

def _exact_held(x):
    """What 8 bits hold of fp64 [rows, cols]: each block's power from its largest magnitude, each value to the nearest of e4m3's
    (three digits behind the leading one, 2^-9 the smallest step), halves to the even one."""
    rows, cols = x.shape
    blocks = -(-cols // 128)
    full = x.new_zeros(rows, blocks * 128)
    full[:, :cols] = x
    full = full.reshape(rows, blocks, 128)
    digits, power = torch.frexp(full.abs().amax(2))              # largest = digits 2^power, digits in [1/2, 1); 448 = 7/8 2^9
    e = torch.where(digits > 0.875, power - 8, power - 9).clamp_min(-127)
    e = torch.where(digits == 0, torch.full_like(e, -127), e)[:, :, None]
    v = torch.ldexp(full, -e)
    step = torch.ldexp(torch.ones_like(v), torch.frexp(v)[1].clamp_min(-5) - 4)
    return torch.ldexp(torch.round(v / step) * step, e).reshape(rows, -1)[:, :cols]


def _exact_values(m):
    """fp64 values of a matrix in 8 bits, byte by byte from the layout's definition."""
    codes, scales, cols = m
    rows = codes.shape[0]
    r = torch.arange(rows, device=codes.device)[:, None]
    b = torch.arange(cols, device=codes.device)[None, :] // 128
    at = ((b // 4) * (-(-rows // 128)) + r // 128) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4
    code = codes[:, :cols].long()
    field, digits = (code >> 3) & 15, (code & 7).double()
    size = torch.where(field == 0, digits / 8 * 2.0 ** -6, torch.ldexp(1.0 + digits / 8, field - 7))
    return torch.ldexp(torch.where(code >= 128, -size, size), scales[at].long() - 127)


def _exact_act(g, gelu):
    """share, act' and a mark where 64 bits cannot tell the share, always below 1, from 1."""
    y = GELU_A * (g + GELU_B * g ** 3) if gelu else g
    dy = GELU_A * (1 + 3 * GELU_B * g ** 2) if gelu else 1.0
    share = 1 / (1 + torch.exp(-y))
    slope = share + g * share / (1 + torch.exp(y)) * dy
    return share, slope, share == 1, torch.where(g * dy > 1, 1, -1)


def _exact_next(v, ones, step):
    """v, and where a factor of it was rounded to 1, the number next to v on the side that step (1 away from 0, -1 towards it) says."""
    side = torch.where(torch.as_tensor(step, device=v.device) > 0, torch.sign(v) * math.inf, 0.0)
    return torch.where(ones & (v != 0), torch.nextafter(v, side), v)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "keep":
        return {"read": _exact_held(s["x"][:, :case["cols"]].double())}
    if kind == "product":
        return {"c": torch.einsum("ik,jk->ij", _exact_values(s["a"]), _exact_values(s["b"]))}
    if kind == "weight_grad":
        a, b = _exact_held(s["dy"].double().t()), _exact_held(_exact_values(s["kept"]).t())
        return {"dw": torch.einsum("ir,jr->ij", a, b)}
    x = _exact_values(s["x"])
    if kind == "gated_fwd":
        g = torch.einsum("rd,fd->rf", x, _exact_values(s["gate_w"]))
        u = torch.einsum("rd,fd->rf", x, _exact_values(s["up_w"]))
        share, _, ones, _ = _exact_act(g, case["gelu"])
        h = _exact_next(g * share * u, ones, -1)
        return {"h": _exact_held(h), "gate": _exact_held(g), "up": _exact_held(u)} if case["kept"] else {"h": h}
    g, u, dh = _exact_values(s["gate"]), _exact_values(s["up"]), s["dh"].double()
    share, slope, ones, side = _exact_act(g, case["gelu"])
    dg = _exact_next(dh * u * slope, ones & (slope == 1), side)
    du, h = _exact_next(dh * (g * share), ones, -1), _exact_next(g * share * u, ones, -1)
    dx = torch.einsum("rf,df->rd", _exact_held(dg), _exact_values(s["gate_wt"]))
    dx += torch.einsum("rf,df->rd", _exact_held(du), _exact_values(s["up_wt"]))
    x_t = _exact_held(x.t())
    weight = lambda v: torch.einsum("fr,dr->fd", _exact_held(v.t()), x_t)
    return {"dx": dx, "dgate_w": weight(dg), "dup_w": weight(du),
            "ddown_w": torch.einsum("dr,fr->df", _exact_values(s["dy_t"]), _exact_held(h.t()))}
