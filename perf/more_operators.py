"""What stands around the dense layers of a residual block: the cases on which speed and precision are measured, and the
operators' plain form in elementary torch operations.

  norm           the end of a block and the start of the next: x' = a x + gate norm(h), y = norm(x')
  norm_backward  gradients of that with respect to x, h, the gate and the norms' weights
  dropout        a mask from a counter-based generator, never stored; where asked for with a residual and the 8-bit checkpoint of the result
  mx4            a tensor in microscaled 4-bit floating point (blocks of 32 under a power of two) and read back
  linear_mx4     y = act(x w^T + b) + r, or act(x w^T + b + r), with both operands in that form; x is brought into it within the call
"""
import math

import numpy as np
import torch

#: False: run() computes the plain form.  True: run() calls the library's operators.
own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6
BLOCK = 32                                     # values of a row that share a scale, in 8 bits as in 4
WIDE = 128                                     # columns that rows in 4 bits are padded to


def _norm(name, M, N, dtype, post="rms", pre="rms", gate="columns", groups=1, bias=False, a=1.0, gap=0, op="norm"):
    return {"name": name, "op": op, "M": M, "N": N, "dtype": dtype, "post": post, "pre": pre, "gate": gate, "groups": groups,
            "bias": bias, "a": a, "gap": gap}


def _dropout(name, M, N, dtype, p, residual=False, ckpt=False, gap=0):
    return {"name": name, "op": "dropout", "M": M, "N": N, "dtype": dtype, "p": p, "residual": residual, "ckpt": ckpt, "gap": gap}


def _mx4(name, M, N, dtype, gap=0):
    return {"name": name, "op": "mx4", "M": M, "N": N, "dtype": dtype, "gap": gap}


def _linear(name, M, N, K, dtype, act="none", bias=True, residual="none", gap=0):
    return {"name": name, "op": "linear_mx4", "M": M, "N": N, "K": K, "dtype": dtype, "act": act, "bias": bias,
            "residual": residual, "gap": gap}


def listed():
    return [
        # between two blocks for a single token while serving: the latency of a call
        _norm("norm_token_bf16", 1, 4096, "bf16"),
        # between two blocks in training
        _norm("norm_train_bf16", 8192, 4096, "bf16", a=0.5),
        # odd sizes, rows that are slices of wider ones, a gate for each of 33 samples, means taken off
        _norm("norm_samples_f16", 1023, 1001, "f16", "layer", "layer", "groups", 33, True, gap=3),
        # gradients between two blocks in training
        _norm("norm_backward_train_bf16", 8192, 4096, "bf16", a=0.5, op="norm_backward"),
        # gradients of a gate for each of five samples, odd sizes, 32 bits
        _norm("norm_backward_samples_f32", 645, 1001, "f32", "layer", "layer", "groups", 5, True, op="norm_backward"),
        # a block's hidden layer in training
        _dropout("dropout_train_bf16", 16384, 8192, "bf16", 0.1),
        # onto a residual, odd sizes, slices of wider rows, with what the next layer's gradient reads
        _dropout("dropout_checkpoint_f16", 1023, 1001, "f16", 0.5, True, True, gap=3),
        # weights of a small classifier brought into 4 bits
        _mx4("mx4_small_f32", 1000, 512, "f32"),
        # a block's hidden layer into 4 bits and back
        _mx4("mx4_large_bf16", 16384, 8192, "bf16"),
        # hidden layer for a single token while serving: bound by reading the weights
        _linear("linear_token_bf16", 1, 4096, 4096, "bf16", act="gelu_tanh"),
        # odd sizes, rows that are slices of wider ones, residual before the activation
        _linear("linear_ragged_f16", 1023, 777, 1001, "f16", act="silu", residual="first", gap=3),
        # the widening layer of a block on a long prompt
        _linear("linear_up_bf16", 8192, 16384, 4096, "bf16", act="gelu"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _extent(rng, lo, hi):
    n = _log_int(rng, lo, hi)
    unit = rng.choice([1, 8, 64, 64])          # most layers' extents are multiples of 64, some of nothing
    return max(lo, n // unit * unit)


def draw(rng):
    """One more case: rows from a single token to a training batch, rows' lengths from a small head to a wide block."""
    op = rng.choice(["norm", "norm", "norm_backward", "dropout", "mx4", "linear_mx4", "linear_mx4", "linear_mx4"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    M, N = _log_int(rng, 1, 16384), _extent(rng, 64, 16384)
    if rng.random() < 0.4:
        M = 2 ** int(round(math.log2(M)))
    gap = rng.choice([0, 0, 0, 8, 3])
    if op == "linear_mx4":
        K = _extent(rng, 64, 25088)
        while 2.0 * M * N * K > 1.0e12 or M * max(N, K) > 1.2e8 or N * K > 1.2e8:
            if M > 64:
                M = M * 3 // 4
            elif N >= K:
                N = N * 3 // 4
            else:
                K = K * 3 // 4
        d = _linear("", M, N, K, dtype, rng.choice(["none", "relu", "silu", "gelu", "gelu_tanh"]), rng.random() < 0.8,
                    rng.choice(["none", "none", "after", "first"]), gap)
    else:
        most = 3.0e7 if op.startswith("norm") else 6.0e7
        while M * N > most:
            M = M * 3 // 4
        if op.startswith("norm"):
            gate, groups = rng.choice(["none", "columns", "groups"]), 1
            if gate == "groups":
                groups = _log_int(rng, 1, min(M, 64))
                M = M // groups * groups
            post, pre = rng.choice([("rms", "rms"), ("rms", "rms"), ("layer", "layer"), ("none", "rms"), ("none", "layer"), ("rms", "none")])
            d = _norm("", M, N, dtype, post, pre, gate, groups, rng.random() < 0.5, rng.choice([1.0, 0.5, 0.7]), gap, op)
        elif op == "dropout":
            d = _dropout("", M, N, dtype, round(rng.uniform(0.05, 0.6), 2), rng.random() < 0.4, rng.random() < 0.4, gap)
        else:
            d = _mx4("", M, N, dtype, gap)
    del d["name"]
    return d


# ---- inputs ----------------------------------------------------------------------------------------------------

def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _wide(t, dtype, gap):
    """t in `dtype`, its rows `gap` values apart."""
    wide = torch.empty((t.shape[0], t.shape[1] + gap), device="cuda", dtype=TYPES[dtype])
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def _activations(g, M, K, dtype, gap=0):
    """Rows of a hidden state: centred, a few columns far larger than the rest."""
    x = _normal(g, M, K)
    x *= torch.where(torch.rand((K,), generator=g, device="cuda") < 0.01, 8.0, 1.0)
    return _wide(x, dtype, gap)


def _to_mx4(x):
    """(codes, scales) of x [rows][cols]: two codes a byte, the even column's in the low half; rows padded to 128 columns."""
    rows, cols = x.shape
    nb = -(-cols // WIDE) * WIDE // BLOCK
    v = torch.zeros((rows, nb * BLOCK), device=x.device, dtype=torch.float32)
    v[:, :cols] = x
    v = v.view(rows, nb, BLOCK)
    most = v.abs().amax(2)
    bad = ~v.isfinite().all(2)
    # the least e with most <= 7 2^e: most = f 2^p with f in [0.5, 1), and 7 = 0.875 * 2^3
    f, p = torch.frexp(torch.where(bad, 1.0, most))
    e = torch.where(f <= 0.875, p - 3, p - 2).clamp(min=-127)
    e = torch.where(most == 0, -127, e)
    half = torch.div(e, 2, rounding_mode="floor")           # 2^-e in two factors: 2^127 is a value, 2^-127 a small one
    one = torch.ones_like(most)
    u = v * torch.ldexp(one, -half).unsqueeze(2) * torch.ldexp(one, half - e).unsqueeze(2)
    a = u.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = (torch.round(a / step) * step).clamp(max=6.0)
    code = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4))      # 0 .5 1 1.5 2 3 4 6
    code = torch.where(bad.unsqueeze(2), 0.0, code + 8 * (torch.signbit(v) & (a > 0)))
    code = code.to(torch.uint8).view(rows, -1, 2)
    return code[:, :, 0] + 16 * code[:, :, 1], torch.where(bad, 255, e + 127).to(torch.uint8)


def _of_mx4(codes, scales, cols):
    rows = codes.shape[0]
    code = torch.stack([codes & 15, codes >> 4], 2).view(rows, -1)[:, :cols].long()
    level = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    e = scales.to(torch.int32) - 127
    half = torch.div(e, 2, rounding_mode="floor")
    one = torch.ones_like(e, dtype=torch.float32)
    value = level[code]
    for part in (half, e - half):
        value = value * torch.ldexp(one, part).repeat_interleave(BLOCK, 1)[:, :cols]
    return torch.where((scales == 255).repeat_interleave(BLOCK, 1)[:, :cols], math.nan, value)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, M, N, dtype, gap = case["op"], case["M"], case["N"], case["dtype"], case["gap"]
    T = TYPES[dtype]
    state = {"case": case}
    if op == "mx4":
        state["x"] = _activations(g, M, N, dtype, gap)
    elif op == "dropout":
        state["x"] = _activations(g, M, N, dtype, gap)
        state["r"] = _wide(_normal(g, M, N), dtype, gap) if case["residual"] else None
        state["seed"], state["offset"] = seed * 0x9E3779B97F4A7C15 % 2 ** 64, 3 + seed % 1000
    elif op == "linear_mx4":
        K = case["K"]
        state["x"] = _activations(g, M, K, dtype, gap)
        # weights are brought into 4 bits once, when a model is loaded
        state["w"] = _to_mx4((_normal(g, N, K) * math.sqrt(2.0 / K)).to(T).float())
        state["b"] = (_normal(g, N) * 0.1).to(T) if case["bias"] else None
        state["r"] = _normal(g, M, N).to(T) if case["residual"] != "none" else None
    else:
        state["x"] = _activations(g, M, N, dtype, gap)
        state["h"] = _wide(_normal(g, M, N) * 0.5 + 0.1, dtype, gap)

        def column(there, level, spread):
            return (level + spread * _normal(g, N)).to(T) if there else None
        state["wp"], state["bp"] = column(case["post"] != "none", 1.0, 0.2), column(case["post"] != "none" and case["bias"], 0.0, 0.1)
        state["w"], state["b"] = column(case["pre"] != "none", 1.0, 0.2), column(case["pre"] != "none" and case["bias"], 0.0, 0.1)
        state["gate"] = None
        if case["gate"] == "columns":
            state["gate"] = (0.5 + 0.2 * _normal(g, N)).to(T)
        elif case["gate"] == "groups":
            state["gate"] = (0.5 + 0.2 * _normal(g, case["groups"], N)).to(T)
        if op == "norm_backward":                  # x is the x' that the forward pass has left
            state["dx"] = _wide(_normal(g, M, N) * 0.02, dtype, gap)
            state["dy"] = _wide(_normal(g, M, N) * 0.02, dtype, gap) if case["pre"] != "none" else None
    return state


# ---- the plain form --------------------------------------------------------------------------------------------

def _hat(v, kind):
    """(v normalised, what it was multiplied with)."""
    if kind == "none":
        return v, torch.ones_like(v[:, :1])
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    r = 1 / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)
    return v * r, r


def _through_hat(d, hat, r, kind):
    """The gradient with respect to v of a row whose normalised form has the gradient d."""
    if kind == "none":
        return d
    d = d - hat * (d * hat).mean(1, keepdim=True) - (d.mean(1, keepdim=True) if kind == "layer" else 0.0)
    return d * r


def _affine(hat, w, b):
    y = hat if w is None else hat * w.float()
    return y if b is None else y + b.float()


def _gate_rows(gate, M):
    if gate is None or gate.dim() == 1:
        return 1.0 if gate is None else gate.float()
    return gate.float().repeat_interleave(M // gate.shape[0], 0)


def _plain_norm(s):
    c = s["case"]
    T = TYPES[c["dtype"]]
    p = _affine(_hat(s["h"].float(), c["post"])[0], s["wp"], s["bp"])
    x = (c["a"] * s["x"].float() + _gate_rows(s["gate"], c["M"]) * p).to(T)
    if c["pre"] == "none":
        return {"x": x}
    # the norm of x' as it is stored
    return {"x": x, "y": _affine(_hat(x.float(), c["pre"])[0], s["w"], s["b"]).to(T)}


def _plain_norm_backward(s):
    c = s["case"]
    T, M, N = TYPES[c["dtype"]], c["M"], c["N"]
    out = {}
    d = s["dx"].float()
    if c["pre"] != "none":
        hat, r = _hat(s["x"].float(), c["pre"])
        dy = s["dy"].float()
        d = d + _through_hat(dy * s["w"].float(), hat, r, c["pre"])
        out["dw"] = (dy * hat).sum(0).to(T)
        if s["b"] is not None:
            out["db"] = dy.sum(0).to(T)
    out["dx"] = (c["a"] * d).to(T)
    hat, r = _hat(s["h"].float(), c["post"])
    if s["gate"] is not None:
        dg = d * _affine(hat, s["wp"], s["bp"])
        out["dgate"] = (dg.sum(0) if s["gate"].dim() == 1 else dg.view(c["groups"], -1, N).sum(1)).to(T)
    d = d * _gate_rows(s["gate"], M)
    if c["post"] != "none":
        out["dwp"] = (d * hat).sum(0).to(T)
        if s["bp"] is not None:
            out["dbp"] = d.sum(0).to(T)
        d = _through_hat(d * s["wp"].float(), hat, r, c["post"])
    out["dh"] = d.to(T)
    return out


def _random_words(groups, seed, offset, device):
    """Philox4x32 with ten rounds (Salmon, Moraes, Dror, Shaw 2011): four words of 32 bits for each of the counters 0 ... groups - 1."""
    low = 0xffffffff
    at = torch.arange(groups, device=device, dtype=torch.int64)
    c = [at & low, at >> 32, torch.full_like(at, offset & low), torch.full_like(at, offset >> 32)]
    k = [seed & low, seed >> 32]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57          # (the low 64 bits)
        c = [((b >> 32) & low) ^ c[1] ^ k[0], b & low, ((a >> 32) & low) ^ c[3] ^ k[1], a & low]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    return c


def _stored(x):
    """What the 8-bit checkpoint of x holds (perf/operators.py: the same blocks)."""
    rows, cols = x.shape
    lo, hi = (-24, 10) if x.dtype == torch.float16 else (-126, 122)
    nb = -(-cols // BLOCK)
    v = torch.zeros((rows, nb * BLOCK), device=x.device, dtype=torch.float32)
    v[:, :cols] = x
    v = v.view(rows, nb, BLOCK)
    f, p = torch.frexp(v.abs().amax(2))
    e = torch.where(f <= 0.9921875, p - 7, p - 6).clamp(lo, hi)
    unit = torch.ldexp(torch.ones_like(f), e).unsqueeze(2)
    return (torch.round(v / unit) * unit).view(rows, -1)[:, :cols].to(x.dtype)


def _plain_dropout(s):
    c = s["case"]
    M, N = c["M"], c["N"]
    least = round(c["p"] * 65536)
    per = -(-N // 8)
    words = _random_words(M * per, s["seed"], s["offset"], s["x"].device)
    keep = torch.stack([(w >> shift & 0xffff) >= least for w in words for shift in (0, 16)], 1).view(M, per * 8)[:, :N]
    y = torch.where(keep, s["x"].float() * (65536.0 / (65536 - least)), 0.0)
    if s["r"] is not None:
        y = y + s["r"].float()
    y = y.to(TYPES[c["dtype"]])
    return {"y": y, "stored": _stored(y)} if c["ckpt"] else y


def _act(z, name):
    if name == "relu":
        return torch.where(z > 0, z, torch.where(z <= 0, 0.0, z))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _plain_linear(s):
    c = s["case"]
    x = _of_mx4(*_to_mx4(s["x"].float()), c["K"])
    z = torch.mm(x, _of_mx4(*s["w"], c["K"]).t())
    if s["b"] is not None:
        z = z + s["b"].float()
    if c["residual"] == "first":
        z = z + s["r"].float()
    y = _act(z, c["act"])
    if c["residual"] == "after":
        y = y + s["r"].float()
    return y.to(TYPES[c["dtype"]])


def _plain(state):
    c = state["case"]
    if c["op"] == "mx4":
        return _of_mx4(*_to_mx4(state["x"].float()), c["N"]).to(TYPES[c["dtype"]])
    return {"norm": _plain_norm, "norm_backward": _plain_norm_backward, "dropout": _plain_dropout,
            "linear_mx4": _plain_linear}[c["op"]](state)


# ---- the library's operators ---------------------------------------------------------------------------------------

def _own(s):
    from paper_2012_15667_amd import binding as B
    c = s["case"]
    T = TYPES[c["dtype"]]
    if c["op"] == "mx4":
        return B.mx4_unpack(B.mx4_pack(s["x"]), T)
    if c["op"] == "linear_mx4":
        return B.linear_mx4(s["x"], B.Mx4(s["w"][0], s["w"][1], c["K"]), s["b"], act=c["act"], residual=s["r"],
                            residual_first=c["residual"] == "first")
    if c["op"] == "dropout":
        if not c["ckpt"]:
            return B.dropout(s["x"], c["p"], s["seed"], s["offset"], residual=s["r"])
        y, stored = B.dropout(s["x"], c["p"], s["seed"], s["offset"], residual=s["r"], checkpoint=True)
        return {"y": y, "stored": B.checkpoint_unpack(stored, T)}
    if c["op"] == "norm":
        n = B.block_norm(s["x"], s["h"], post=c["post"], post_weight=s["wp"], post_bias=s["bp"], gate=s["gate"], scale=c["a"],
                         pre=c["pre"], pre_weight=s["w"], pre_bias=s["b"], eps=EPS)
        return {"x": n.x} if c["pre"] == "none" else {"x": n.x, "y": n.y}
    n = B.block_norm_backward(s["dy"], s["dx"], s["x"], s["h"], post=c["post"], post_weight=s["wp"], post_bias=s["bp"],
                              gate=s["gate"], scale=c["a"], pre=c["pre"], pre_weight=s["w"], pre_bias=s["b"], eps=EPS)
    all_of = {"dw": n.dpre_weight, "db": n.dpre_bias, "dx": n.dx, "dgate": n.dgate, "dwp": n.dpost_weight, "dbp": n.dpost_bias, "dh": n.dh}
    return {k: v for k, v in all_of.items() if v is not None}


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    """Inputs read once, outputs written once; what is stored in 8 or 4 bits and read back counts both ways."""
    M, N, b, op = case["M"], case["N"], BYTES[case["dtype"]], case["op"]
    if op == "mx4":
        return {"bytes": 2 * b * M * N + 2 * M * (-(-N // 2) + -(-N // BLOCK)), "flops": 0}
    if op == "dropout":
        n = (3 if case["residual"] else 2) * b * M * N
        if case["ckpt"]:
            n += 2 * M * (N + -(-N // BLOCK)) + b * M * N
        return {"bytes": n, "flops": 0}
    if op == "linear_mx4":
        K = case["K"]
        n = b * (M * K + M * N + (N if case["bias"] else 0) + (M * N if case["residual"] != "none" else 0))
        return {"bytes": n + N * (-(-K // 2) + -(-K // BLOCK)), "flops": 2 * M * N * K}
    rows = 3 + (case["pre"] != "none") + (2 if op == "norm_backward" else 0)
    columns = {"none": 0, "columns": 1, "groups": case["groups"]}[case["gate"]]
    columns += ((case["post"] != "none") + (case["pre"] != "none")) * (2 if case["bias"] else 1)
    return {"bytes": b * N * (rows * M + columns * (2 if op == "norm_backward" else 1)), "flops": 0}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------

def _exact_norm_of(v, kind, w, b):
    if kind == "none":
        return v
    var, mean = torch.var_mean(v, 1, correction=0, keepdim=True)
    y = v / torch.sqrt(v.square().mean(1, keepdim=True) + EPS) if kind == "rms" else (v - mean) * (var + EPS) ** -0.5
    return y * w + (0 if b is None else b)


def _exact_norm(c, s):
    t = {k: v.double() for k, v in s.items() if torch.is_tensor(v)}
    p = _exact_norm_of(t["h"], c["post"], t.get("wp"), t.get("bp"))
    g = t.get("gate", torch.ones((), dtype=torch.float64, device="cuda"))
    if g.dim() == 2:
        g = g[torch.arange(c["M"], device="cuda") // (c["M"] // c["groups"])]
    return torch.addcmul(c["a"] * t["x"], g, p)


def _exact_norm_forward(c, s):
    x = _exact_norm(c, s)
    if c["pre"] == "none":
        return {"x": x}
    t = {k: v.double() for k, v in s.items() if torch.is_tensor(v)}
    return {"x": x, "y": _exact_norm_of(x.to(TYPES[c["dtype"]]).double(), c["pre"], t["w"], t.get("b"))}


def _exact_norm_backward(c, s):
    """By differentiation of the forward definition, row by row stored x' taken as the norm's input."""
    names = [k for k in ("wp", "bp", "w", "b", "gate", "h") if s.get(k) is not None]
    leaf = {k: s[k].double().requires_grad_() for k in names}
    # the stored x' is a leaf of its own: its gradient d goes on to x (times a) and through the gate to h
    out = s["x"].double().requires_grad_()
    d = s["dx"].double()
    if c["pre"] != "none":
        y = _exact_norm_of(out, c["pre"], leaf["w"], leaf.get("b"))
        y.backward(s["dy"].double())
        d = d + out.grad
        del y
    sum_ = _exact_norm(c, {"x": torch.zeros_like(d), **leaf})
    sum_.backward(d)
    found = {"dw": leaf.get("w"), "db": leaf.get("b"), "dgate": leaf.get("gate"), "dwp": leaf.get("wp"), "dbp": leaf.get("bp"), "dh": leaf["h"]}
    return {"dx": c["a"] * d, **{k: v.grad for k, v in found.items() if v is not None and v.grad is not None}}


def _exact_keep(M, N, p, seed, offset):
    """The mask by numpy's unsigned arithmetic."""
    per = (N + 7) // 8
    u32, u64 = np.uint32, np.uint64
    i = np.arange(M * per, dtype=u64)
    x0, x1 = (i & u64(2 ** 32 - 1)).astype(u32), (i >> u64(32)).astype(u32)
    x2, x3 = np.full(M * per, offset % 2 ** 32, dtype=u32), np.full(M * per, offset // 2 ** 32, dtype=u32)
    for turn in range(10):
        k0, k1 = u32((seed + turn * 0x9E3779B9) % 2 ** 32), u32((seed // 2 ** 32 + turn * 0xBB67AE85) % 2 ** 32)
        m, n = x0.astype(u64) * u64(0xD2511F53), x2.astype(u64) * u64(0xCD9E8D57)
        x0, x1, x2, x3 = (n >> u64(32)).astype(u32) ^ x1 ^ k0, n.astype(u32), (m >> u64(32)).astype(u32) ^ x3 ^ k1, m.astype(u32)
    halves = np.ascontiguousarray(np.stack([x0, x1, x2, x3], 1)).view("<u2").reshape(M, per * 8)[:, :N]
    return torch.from_numpy(halves >= round(p * 65536)).cuda()


def _exact_mx4(x):
    """The values that x holds in 4 bits: by distance to each of the eight magnitudes."""
    rows, cols = x.shape
    blocks = torch.nn.functional.pad(x.double(), (0, -cols % BLOCK)).unflatten(1, (-1, BLOCK))
    most = blocks.abs().amax(2, keepdim=True)
    e = torch.ceil(torch.log2((most / 7).clamp(min=2.0 ** -140)))
    e = torch.where(7 * torch.exp2(e - 1) >= most, e - 1, e)
    e = torch.where(7 * torch.exp2(e) < most, e + 1, e).clamp(min=-127)
    unit = torch.exp2(e)
    u = blocks.abs() / unit
    level = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    a = torch.zeros_like(u)
    for i in range(7):                          # beyond the middle of two levels, or on it where the upper one is even
        middle = (level[i] + level[i + 1]) / 2
        a = torch.where((u >= middle) if i % 2 else (u > middle), level[i + 1], a)
    return (a * blocks.sign() * unit).flatten(1)[:, :cols].contiguous()


def _exact_act(z, name):
    return {"none": lambda: z, "relu": lambda: z.clamp(min=0), "silu": lambda: z * torch.sigmoid(z), "gelu": lambda: z * torch.special.ndtr(z),
            "gelu_tanh": lambda: z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))}[name]()


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "mx4":
        return _exact_mx4(s["x"])
    if case["op"] == "norm":
        return _exact_norm_forward(case, s)
    if case["op"] == "norm_backward":
        return _exact_norm_backward(case, s)
    if case["op"] == "dropout":
        keep = _exact_keep(case["M"], case["N"], case["p"], s["seed"], s["offset"])
        y = s["x"].double() * keep * (65536 / (65536 - round(case["p"] * 65536)))
        if s["r"] is not None:
            y += s["r"].double()
        # a value beside the middle of two 8-bit values goes to either with its last bit
        return {"y": y, "stored": None} if case["ckpt"] else y
    codes, scales = s["w"]
    levels = np.array([0, 1, 2, 3, 4, 6, 8, 12], dtype=np.float64) / 2
    table = torch.from_numpy(np.concatenate([levels, -levels])).cuda()
    w = torch.empty((codes.shape[0], 2 * codes.shape[1]), dtype=torch.float64, device="cuda")
    w[:, 0::2], w[:, 1::2] = table[(codes % 16).long()], table[(codes // 16).long()]
    w = (w.unflatten(1, (-1, BLOCK)) * torch.exp2(scales.double() - 127).unsqueeze(2)).flatten(1)[:, :case["K"]]
    z = _exact_mx4(s["x"]) @ w.t().contiguous()
    if s["b"] is not None:
        z += s["b"].double()
    if case["residual"] == "first":
        z += s["r"].double()
    y = _exact_act(z, case["act"])
    return y + s["r"].double() if case["residual"] == "after" else y
