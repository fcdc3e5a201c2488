"""A feed-forward block and an output layer with its loss, as the users of ``paper_2112_00709_amd`` call them, and their plain forms.

What lies in front of a network's pseudo-log-likelihoods: the way from one block into the next (norms, gate, residual scale
and residual in one pass), a gated layer (both projections, activation and product), and the log probabilities of given
tokens straight from hidden frames, the logits never kept; each with its gradient.  Rows are frames (batch x time)
throughout; 69120 of them are the 128 utterances of up to 540 frames, 44160 those of mean length, and 3000 outputs are the
pdfs, of this repository's large workload; 128000 tokens are a large vocabulary.

``dtype``: "bf16", "f16" or "f32", the type of activations, weights and gates; ``gap``: the rows are slices of a
tensor that is so many columns wider.
"""
import math

import torch

own = False

EPS = 1e-5
DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}


def listed():
    return [
        # a recogniser that is fed frame by frame: from one block into the next for a single frame, nothing but latency
        dict(name="residual_frame", op="residual_norm", R=1, H=512, dtype="bf16", gap=0, inner="rms", outer="rms", gate="none", residual=True),
        # the same step for a large batch of utterances in training, with a learned scale a column
        dict(name="residual_batch", op="residual_norm", R=69120, H=1024, dtype="bf16", gap=0, inner="rms", outer="rms", gate="vector", residual=True),
        # its backward pass, with a gate for every element and the gradients of both norms' weights
        dict(name="residual_grad_batch", op="residual_norm_grad", R=69120, H=1024, dtype="bf16", gap=0, inner="layer", outer="layer", gate="rows"),
        # a minibatch of short utterances in single precision, an odd width inside a wider tensor
        dict(name="residual_grad_odd", op="residual_norm_grad", R=4811, H=777, dtype="f32", gap=5, inner="rms", outer="layer", gate="vector"),
        # one frame through a gated layer, in a recogniser that is fed frame by frame
        dict(name="gated_frame", op="gated", M=1, N=4096, K=1024, dtype="bf16", act="silu", preact=False, gap=0),
        # a gated layer on a batch of utterances of mean length, in training
        dict(name="gated_batch", op="gated", M=44160, N=2048, K=1024, dtype="bf16", act="silu", preact=True, gap=0),
        # its backward products
        dict(name="gated_grad_batch", op="gated_grad", M=44160, N=2048, K=1024, dtype="bf16", act="silu", gap=0),
        # a minibatch of odd sizes in half precision
        dict(name="gated_grad_odd", op="gated_grad", M=9601, N=1111, K=777, dtype="f16", act="gelu", gap=0),
        # one step of a decoder that scores a given token over a large vocabulary
        dict(name="vocabulary_step", op="logprobs", M=1, V=128000, K=1024, dtype="bf16", gap=0),
        # a token loss over a large vocabulary, a batch of sequences
        dict(name="vocabulary_batch", op="logprobs", M=4095, V=128000, K=2048, dtype="bf16", gap=0),
        # frame cross entropy on an alignment beside the objective, its gradient on a large batch of utterances
        dict(name="frames_grad", op="logprobs_grad", M=69120, V=3000, K=1024, dtype="bf16", gap=0, entropy=True),
        # the gradient of the token loss over the large vocabulary
        dict(name="vocabulary_grad", op="logprobs_grad", M=4095, V=128000, K=2048, dtype="bf16", gap=0, entropy=False),
    ]


# --------------------------------------------------------------------------- more cases of the same ranges

def _log_int(rng, lo, hi):
    n = min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    if n >= 64 and rng.random() < 0.4:      # widths of real layers are often round
        n = min(hi, (n + 63) // 64 * 64)
    return n


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    gap = rng.choice([0, 0, 0, rng.randint(1, 40)])
    slow = 4 if dtype == "f32" else 1
    kind = rng.random()
    if kind < 0.34:
        R, H = _log_int(rng, 1, 69120), _log_int(rng, 16, 8192)
        R = min(R, 69120 * 1024 // H)
        c = dict(op=rng.choice(["residual_norm", "residual_norm_grad"]), R=R, H=H, dtype=dtype, gap=gap, inner=rng.choice(["none", "layer", "rms"]),
                 outer=rng.choice(["none", "layer", "rms", "rms"]), gate=rng.choice(["none", "vector", "rows"]))
        if c["op"] == "residual_norm":
            c["residual"] = rng.random() < 0.8
        return c
    if kind < 0.67:
        grad = rng.random() < 0.5
        M, N, K = _log_int(rng, 1, 69120), _log_int(rng, 16, 4096), _log_int(rng, 16, 4096)
        M = max(1, min(M, 44160 * 2048 * 1024 // (2 if grad else 1) // slow // (N * K)))
        act = rng.choice(["none", "relu", "gelu", "silu", "sigmoid"])
        if grad:
            return dict(op="gated_grad", M=M, N=N, K=K, dtype=dtype, act=act, gap=gap)
        return dict(op="gated", M=M, N=N, K=K, dtype=dtype, act=act, preact=rng.random() < 0.5, gap=gap)
    grad = rng.random() < 0.5
    M, V, K = _log_int(rng, 1, 69120), _log_int(rng, 40, 131072), _log_int(rng, 16, 4096)
    M = max(1, min(M, 69120 * 3000 * 1024 // (2 if grad else 1) // slow // (V * K), 69120 * 3000 // V))
    if grad:
        return dict(op="logprobs_grad", M=M, V=V, K=K, dtype=dtype, gap=gap, entropy=rng.random() < 0.5)
    return dict(op="logprobs", M=M, V=V, K=K, dtype=dtype, gap=gap)


# --------------------------------------------------------------------------- inputs

class _Source:
    """Normal and uniform numbers on the GPU from a seed."""

    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda").manual_seed(seed * 2 + 1)

    def rows(self, rows, width, dtype, gap=0, scale=1.0, shift=None):
        x = torch.randn((rows, width + gap), device="cuda", generator=self.gen)
        x *= scale
        if shift is not None:
            x += shift
        return x.to(dtype)[:, :width]

    def normal(self, *shape):
        return torch.randn(shape, device="cuda", generator=self.gen)

    def uniform(self, *shape):
        return torch.rand(shape, device="cuda", generator=self.gen)

    def below(self, n, count):
        return torch.randint(0, n, (count,), device="cuda", generator=self.gen, dtype=torch.int32)


def prepare(case, seed):
    s, t, op = _Source(seed), DTYPE[case["dtype"]], case["op"]
    c = dict(case=case, inner_weight=None, inner_bias=None, weight=None, bias=None, gate=None, residual=None, scale=0.7)
    if op in ("residual_norm", "residual_norm_grad"):
        R, H = case["R"], case["H"]
        c["h"] = s.rows(R, H, t, case["gap"], 0.8, 0.3 * s.normal(R, 1))
        if case["inner"] != "none":
            c["inner_weight"] = 1 + 0.2 * s.normal(H)
            c["inner_bias"] = 0.1 * s.normal(H) if case["inner"] == "layer" else None
        if case["outer"] != "none":
            c["weight"] = 1 + 0.2 * s.normal(H)
            c["bias"] = 0.1 * s.normal(H) if case["outer"] == "layer" else None
        if case["gate"] == "vector":
            c["gate"] = 0.5 + 0.2 * s.normal(H)
        elif case["gate"] == "rows":
            c["gate"] = s.rows(R, H, t, case["gap"], 0.3, 0.5)
        c["residual"] = s.rows(R, H, t, case["gap"], 1.5) if case.get("residual", True) else None
        if op == "residual_norm_grad":              # what the forward pass has handed over
            c["s"], _, c["stats"] = _residual_norm(c)
            c["ds"] = s.rows(R, H, t, case["gap"], 0.1)
            c["dy"] = s.rows(R, H, t, case["gap"], 0.1) if case["outer"] != "none" else None
    elif op in ("gated", "gated_grad"):
        M, N, K = case["M"], case["N"], case["K"]
        c["x"] = s.rows(M, K, t, case["gap"])
        c["weight"] = s.rows(2 * N, K, t, 0, K ** -0.5)
        if op == "gated":
            c["bias"] = 0.1 * s.normal(2 * N)
        else:
            c["preact"] = s.rows(M, 2 * N, t, case["gap"])
            c["dy"] = s.rows(M, N, t, case["gap"], 0.1)
    else:
        M, V, K = case["M"], case["V"], case["K"]
        x = s.normal(M, K + case["gap"])
        c["tokens"] = s.below(V, M)
        if M > 1:                                   # padded frames hold anything
            pad = s.uniform(M) < 0.1
            c["tokens"] = torch.where(pad, torch.full_like(c["tokens"], -1), c["tokens"])
            x.masked_fill_((pad & (s.uniform(M) < 0.5))[:, None], math.nan)
        c["x"] = x.to(t)[:, :K]
        c["weight"] = s.rows(V, K, t, 0, 2 * K ** -0.5)
        c["bias"] = 0.5 * s.normal(V)
        if op == "logprobs_grad":
            c["g_logprobs"] = -1 - 0.1 * s.normal(M)                                             # a sum over frames, as the objective is
            c["g_entropy"] = -0.1 - 0.01 * s.normal(M) if case["entropy"] else None
            _, c["entropy"], c["logz"] = _logprobs(c["x"], c["weight"], c["bias"], c["tokens"])
    return c


# --------------------------------------------------------------------------- the plain forms

def _norm(x, kind, weight, bias):
    """-> the normalised rows, mean, 1 / deviation."""
    mean, rstd = torch.zeros_like(x[:, 0]), torch.ones_like(x[:, 0])
    if kind == "none":
        return x, mean, rstd
    if kind == "layer":
        mean = x.mean(1)
    d = x - mean[:, None]
    rstd = (d.square().mean(1) + EPS).rsqrt()
    y = d * rstd[:, None] * weight
    return y if bias is None else y + bias, mean, rstd


def _residual_norm(c):
    case, h = c["case"], c["h"]
    u, m1, r1 = _norm(h.float(), case["inner"], c["inner_weight"], c["inner_bias"])
    if c["gate"] is not None:
        u = u * c["gate"].float()
    s = u * c["scale"]
    if c["residual"] is not None:
        s = s + c["residual"].float()
    y, m2, r2 = _norm(s, case["outer"], c["weight"], c["bias"])
    return s.to(h.dtype), None if case["outer"] == "none" else y.to(h.dtype), torch.stack([m1, r1, m2, r2])


def _norm_grad(g, xh, rstd, kind):
    if kind == "none":
        return g
    d = g - xh * (g * xh).mean(1, keepdim=True)
    if kind == "layer":
        d = d - g.mean(1, keepdim=True)
    return d * rstd[:, None]


def _residual_norm_grad(c):
    case, t = c["case"], c["h"].dtype
    m1, r1, m2, r2 = c["stats"]
    d = c["ds"].float()
    dw = db = dw1 = db1 = dgate = None
    if case["outer"] != "none":
        dy, xh = c["dy"].float(), (c["s"].float() - m2[:, None]) * r2[:, None]
        dw, db = (dy * xh).sum(0), dy.sum(0)
        d = d + _norm_grad(dy * c["weight"], xh, r2, case["outer"])
    xh = (c["h"].float() - m1[:, None]) * r1[:, None]
    du = d * c["scale"]
    if c["gate"] is not None:
        u = xh
        if case["inner"] != "none":
            u = xh * c["inner_weight"] + (0.0 if c["inner_bias"] is None else c["inner_bias"])
        dgate = du * u
        dgate = dgate.sum(0) if case["gate"] == "vector" else dgate.to(t)
        du = du * c["gate"].float()
    g = du
    if case["inner"] != "none":
        dw1, db1 = (du * xh).sum(0), du.sum(0)
        g = du * c["inner_weight"]
    return _norm_grad(g, xh, r1, case["inner"]).to(t), d.to(t), dgate, dw1, db1, dw, db


def _act(z, name):
    if name == "relu":
        return torch.where(z > 0, z, 0.0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "sigmoid":
        return 1 / (1 + torch.exp(-z))
    return z


def _act_slope(z, name):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    s = 1 / (1 + torch.exp(-z))
    return s * (1 - s) if name == "sigmoid" else s * (1 + z * (1 - s))


def _gated(x, weight, bias, act, preact):
    z = x.float() @ weight.float().t() + bias
    g, u = z.chunk(2, dim=1)
    y = (_act(g, act) * u).to(x.dtype)
    return (y, z.to(x.dtype)) if preact else y


def _gated_grad(dy, x, weight, preact, act):
    g, u = preact.float().chunk(2, dim=1)
    d = dy.float()
    dz = torch.cat([d * u * _act_slope(g, act), d * _act(g, act)], dim=1)
    return (dz @ weight.float()).to(x.dtype), (dz.t() @ x.float()).to(weight.dtype), dz.sum(0)


def _logits(x, weight, bias, live):
    return torch.where(live[:, None], x.float(), 0.0) @ weight.float().t() + bias


def _logprobs(x, weight, bias, tokens):
    live = tokens >= 0
    z = _logits(x, weight, bias, live)
    m = z.max(1).values
    d = z - m[:, None]
    e = torch.exp(d)
    total = e.sum(1)
    logz = m + torch.log(total)
    given = z.gather(1, tokens.clamp_min(0).long()[:, None])[:, 0]
    entropy = torch.log(total) - (e * d).sum(1) / total
    zero = torch.zeros_like(logz)
    return torch.where(live, given - logz, zero), torch.where(live, entropy, zero), torch.where(live, logz, zero)


def _logprobs_grad(x, weight, bias, tokens, logz, entropy, g_logprobs, g_entropy):
    live = tokens >= 0
    logp = _logits(x, weight, bias, live) - logz[:, None]
    p = torch.exp(logp)
    d = -p * g_logprobs[:, None]
    if g_entropy is not None:
        d -= p * (logp + entropy[:, None]) * g_entropy[:, None]
    d.scatter_add_(1, tokens.clamp_min(0).long()[:, None], g_logprobs[:, None])
    d = torch.where(live[:, None], d, 0.0)
    xf = torch.where(live[:, None], x.float(), 0.0)
    return (d @ weight.float()).to(x.dtype), (d.t() @ xf).to(weight.dtype), d.sum(0)


def run(c):
    case, op = c["case"], c["case"]["op"]
    if own:
        from paper_2112_00709_amd import layers as fl
        if op == "residual_norm":
            return fl.fb_residual_norm(c["h"], c["residual"], c["gate"], scale=c["scale"], inner=case["inner"], inner_weight=c["inner_weight"],
                                       inner_bias=c["inner_bias"], outer=case["outer"], weight=c["weight"], bias=c["bias"], eps=EPS, want_stats=True)
        if op == "residual_norm_grad":
            return fl.fb_residual_norm_grad(c["ds"], c["dy"], c["h"], c["s"], c["stats"], c["gate"], scale=c["scale"], inner=case["inner"],
                                            inner_weight=c["inner_weight"], inner_bias=c["inner_bias"], outer=case["outer"], weight=c["weight"])
        if op == "gated":
            return fl.fb_gated_affine(c["x"], c["weight"], c["bias"], activation=case["act"], want_preact=case["preact"])
        if op == "gated_grad":
            return fl.fb_gated_affine_grad(c["dy"], c["x"], c["weight"], c["preact"], activation=case["act"])
        if op == "logprobs":
            return fl.fb_affine_logprobs(c["x"], c["weight"], c["tokens"], c["bias"])
        return fl.fb_affine_logprobs_grad(c["x"], c["weight"], c["tokens"], c["logz"], c["entropy"], c["g_logprobs"], c["g_entropy"], c["bias"])
    if op == "residual_norm":
        return _residual_norm(c)
    if op == "residual_norm_grad":
        return _residual_norm_grad(c)
    if op == "gated":
        return _gated(c["x"], c["weight"], c["bias"], case["act"], case["preact"])
    if op == "gated_grad":
        return _gated_grad(c["dy"], c["x"], c["weight"], c["preact"], case["act"])
    if op == "logprobs":
        return _logprobs(c["x"], c["weight"], c["bias"], c["tokens"])
    return _logprobs_grad(c["x"], c["weight"], c["bias"], c["tokens"], c["logz"], c["entropy"], c["g_logprobs"], c["g_entropy"])


# --------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    e, op = BYTES[case["dtype"]], case["op"]
    if op in ("residual_norm", "residual_norm_grad"):
        R, H = case["R"], case["H"]
        inner, outer, rows, vector = case["inner"] != "none", case["outer"] != "none", case["gate"] == "rows", case["gate"] == "vector"
        vectors = (case["inner"] == "layer") + inner + outer + vector
        if op == "residual_norm":
            moved = 2 + case["residual"] + rows + outer                          # h, s; residual, gate, y
            return {"bytes": moved * R * H * e + 4 * H * (vectors + (case["outer"] == "layer")) + 16 * R, "flops": (2 + 6 * inner + 6 * outer) * R * H}
        moved = 3 + (inner or case["gate"] != "none") + 2 * outer + 2 * rows     # ds, dh, dresidual; h; dy and s; gate and dgate
        sums = 2 * inner + 2 * outer + vector
        return {"bytes": moved * R * H * e + 4 * H * (vectors + sums) + 16 * R, "flops": (4 + 14 * inner + 14 * outer) * R * H}
    if op in ("gated", "gated_grad"):
        M, N, K = case["M"], case["N"], case["K"]
        if op == "gated":
            return {"bytes": (M * K + 2 * N * K + M * N * (3 if case["preact"] else 1)) * e + 8 * N, "flops": 4 * M * N * K}
        return {"bytes": (2 * M * K + 4 * N * K + 3 * M * N) * e + 8 * N, "flops": 8 * M * N * K}
    M, V, K = case["M"], case["V"], case["K"]
    if op == "logprobs":
        return {"bytes": (M * K + V * K) * e + 4 * V + 16 * M, "flops": 2 * M * V * K}
    return {"bytes": 2 * (M * K + V * K) * e + 8 * V + (20 if case["entropy"] else 12) * M, "flops": 6 * M * V * K}


# --------------------------------------------------------------------------- the definitions in 64 bits

def _exact_norm(x, kind, weight, bias):
    """Normalised rows in 64 bits, -> (y, xh, mean, deviation)."""
    D = torch.float64
    n = x.shape[0]
    if kind == "none":
        return x, x, x.new_zeros(n), x.new_ones(n)
    if kind == "layer":
        var, mean = torch.var_mean(x, dim=1, correction=0)
    else:
        var, mean = torch.linalg.vector_norm(x, dim=1) ** 2 / x.shape[1], x.new_zeros(n)
    dev = torch.sqrt(var + EPS)
    xh = (x - mean.unsqueeze(1)) / dev.unsqueeze(1)
    y = xh * weight.to(D)
    return y + bias.to(D) if bias is not None else y, xh, mean, dev


def _exact_back(v, xh, dev, kind):
    """v through the Jacobian of a norm without weights, (I - [1 1' / H] - xh xh' / H) / dev."""
    if kind == "none":
        return v
    H = v.shape[1]
    along = torch.linalg.vecdot(v, xh).unsqueeze(1) / H
    level = v.sum(1, keepdim=True) / H if kind == "layer" else 0.0
    return (v - level - along * xh) / dev.unsqueeze(1)


def exact(case, seed):
    c, op, D = prepare(case, seed), case["op"], torch.float64
    if op == "residual_norm":
        u, _, m1, d1 = _exact_norm(c["h"].to(D), case["inner"], c["inner_weight"], c["inner_bias"])
        factor = c["scale"] if c["gate"] is None else c["gate"].to(D) * c["scale"]
        s = torch.mul(u, factor)
        if c["residual"] is not None:
            s = torch.add(c["residual"].to(D), s)
        y, _, m2, d2 = _exact_norm(s, case["outer"], c["weight"], c["bias"])
        return s, y if case["outer"] != "none" else None, torch.stack((m1, d1.reciprocal(), m2, d2.reciprocal()))
    if op == "residual_norm_grad":
        mean1, rstd1, mean2, rstd2 = c["stats"].to(D).unbind(0)
        total, dw, db, dgate, dw1, db1 = c["ds"].to(D), None, None, None, None, None
        if case["outer"] != "none":
            dy = c["dy"].to(D)
            at = (c["s"].to(D) - mean2.unsqueeze(1)) * rstd2.unsqueeze(1)
            dw, db = torch.linalg.vecdot(dy, at, dim=0), torch.sum(dy, 0)
            total = total + _exact_back(dy * c["weight"].to(D), at, 1 / rstd2, case["outer"])
        at = (c["h"].to(D) - mean1.unsqueeze(1)) * rstd1.unsqueeze(1)
        back = total * c["scale"]
        if c["gate"] is not None:
            u = at if c["inner_weight"] is None else at * c["inner_weight"].to(D)
            u = u if c["inner_bias"] is None else u + c["inner_bias"].to(D)
            dgate = torch.linalg.vecdot(back, u, dim=0) if case["gate"] == "vector" else back * u
            back = back * c["gate"].to(D)
        if case["inner"] != "none":
            dw1, db1 = torch.linalg.vecdot(back, at, dim=0), torch.sum(back, 0)
            back = back * c["inner_weight"].to(D)
        return _exact_back(back, at, 1 / rstd1, case["inner"]), total, dgate, dw1, db1, dw, db
    if op in ("gated", "gated_grad"):
        N, a = case["N"], case["act"]
        if op == "gated":
            z = torch.addmm(c["bias"].to(D), c["x"].to(D), c["weight"].to(D).t().contiguous())
        else:
            z = c["preact"].to(D)
        g, u = z[:, :N], z[:, N:]
        sig = torch.sigmoid(g)
        value = {"none": lambda: g, "relu": lambda: g.clamp_min(0), "gelu": lambda: g * torch.special.ndtr(g), "silu": lambda: g * sig, "sigmoid": lambda: sig}[a]()
        if op == "gated":
            return (value * u, z) if case["preact"] else value * u
        slope = {"none": lambda: torch.ones_like(g), "relu": lambda: torch.heaviside(g, torch.zeros_like(g)),
                 "gelu": lambda: torch.special.ndtr(g) + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi),
                 "silu": lambda: sig + g * sig * torch.sigmoid(-g), "sigmoid": lambda: sig * torch.sigmoid(-g)}[a]()
        dz = torch.empty_like(z)
        dz[:, :N] = c["dy"].to(D) * slope * u
        dz[:, N:] = c["dy"].to(D) * value
        return torch.mm(dz, c["weight"].to(D)), torch.mm(dz.t().contiguous(), c["x"].to(D)), torch.sum(dz, 0)
    pad = c["tokens"] < 0
    x = c["x"].to(D).masked_fill(pad.unsqueeze(1), 0)
    z = torch.addmm(c["bias"].to(D), x, c["weight"].to(D).t().contiguous())
    at = c["tokens"].long().clamp_min(0).unsqueeze(1)
    if op == "logprobs":
        logp = torch.log_softmax(z, 1)
        logz = torch.logsumexp(z, 1)
        given = torch.take_along_dim(logp, at, 1).squeeze(1)
        entropy = torch.special.entr(logp.exp_()).sum(1)
        return given.masked_fill(pad, 0), entropy.masked_fill(pad, 0), logz.masked_fill(pad, 0)
    p = torch.exp(z - c["logz"].to(D).unsqueeze(1))
    inner = torch.xlogy(p, p) + p * c["entropy"].to(D).unsqueeze(1) if c["g_entropy"] is not None else None
    p.neg_().scatter_add_(1, at, torch.ones_like(at, dtype=D))
    p *= c["g_logprobs"].to(D).unsqueeze(1)
    if inner is not None:
        p -= inner * c["g_entropy"].to(D).unsqueeze(1)
    p.masked_fill_(pad.unsqueeze(1), 0)
    return torch.mm(p, c["weight"].to(D)), torch.mm(p.t().contiguous(), x), torch.sum(p, 0)
