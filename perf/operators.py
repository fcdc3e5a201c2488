"""The operators of a network's last layers, as the users of ``paper_2112_00709_amd`` call them, and their plain forms.

What stands between a network's hidden frames and the objective: the layer norm, the affine layers that make the
pseudo-log-likelihoods (bias, activation and residual in the product's epilogue), and the log probabilities of given
tokens with entropy and best alternatives; each with its gradient.  Rows are frames (batch x time) throughout; 69120
of them are the 128 utterances of up to 540 frames, and 3000 outputs are the pdfs, of this repository's large workload.

``dtype``: "bf16", "f16" or "f32", the type of activations, weights and logits; ``gap``: the rows are slices of a
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
        # a recogniser that is fed frame by frame: one frame's normalisation, nothing but latency
        dict(name="norm_frame", op="layer_norm", R=1, H=512, dtype="bf16", gap=0),
        # the normalisation of a large batch of utterances on the way to the output layer
        dict(name="norm_batch", op="layer_norm", R=69120, H=1024, dtype="bf16", gap=0),
        # its backward pass in a training step, with the gradients of weight and bias
        dict(name="norm_grad_batch", op="layer_norm_grad", R=69120, H=1024, dtype="bf16", gap=0),
        # a minibatch of short utterances in single precision, an odd width inside a wider tensor
        dict(name="norm_grad_odd", op="layer_norm_grad", R=4811, H=777, dtype="f32", gap=5),
        # one frame through a hidden layer with its skip connection, in a recogniser that is fed frame by frame
        dict(name="affine_frame", op="affine", M=1, N=2048, K=2048, dtype="bf16", out="same", act="relu", residual=True, preact=False, gap=0),
        # the output layer on a large batch of utterances: single-precision pseudo-log-likelihoods for the objective
        dict(name="affine_outputs", op="affine", M=69120, N=3000, K=1024, dtype="bf16", out="f32", act="none", residual=False, preact=False, gap=0),
        # a hidden layer in training on a minibatch of odd sizes
        dict(name="affine_odd", op="affine", M=9601, N=1111, K=777, dtype="f16", out="same", act="gelu", residual=True, preact=True, gap=0),
        # the backward products of a hidden layer on a batch of utterances of mean length
        dict(name="affine_grad_batch", op="affine_grad", M=44160, N=2048, K=1024, dtype="bf16", dy="same", act="relu", gap=0),
        # the backward products of a small output layer in single precision (84 outputs, chunks of 150 frames)
        dict(name="affine_grad_small", op="affine_grad", M=9600, N=84, K=512, dtype="f32", dy="f32", act="none", gap=0),
        # one step of a decoder over a large vocabulary: log probability, entropy and the best alternatives
        dict(name="tokens_step", op="logprobs", R=1, V=128000, top=10, dtype="bf16", gap=0),
        # frame log probabilities against an alignment, on the objective's own inputs, a large batch
        dict(name="tokens_frames", op="logprobs", R=69120, V=3000, top=3, dtype="f32", gap=0),
        # the gradient of a token loss with an entropy term over a vocabulary of subwords
        dict(name="tokens_grad", op="logprobs_grad", R=4095, V=32001, top=0, dtype="bf16", gap=0),
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
    kind = rng.random()
    if kind < 0.3:
        R, H = _log_int(rng, 1, 69120), _log_int(rng, 16, 16384)
        R = min(R, 69120 * 1024 // H)
        return dict(op=rng.choice(["layer_norm", "layer_norm_grad"]), R=R, H=H, dtype=dtype, gap=gap)
    if kind < 0.7:
        grad = rng.random() < 0.5
        M, N, K = _log_int(rng, 1, 69120), _log_int(rng, 16, 4096), _log_int(rng, 16, 4096)
        most = 69120 * 3000 * 1024 // (2 if grad else 1) // (4 if dtype == "f32" else 1)
        M = max(1, min(M, most // (N * K)))
        act = rng.choice(["none", "relu", "gelu", "silu"])
        if grad:
            return dict(op="affine_grad", M=M, N=N, K=K, dtype=dtype, dy=rng.choice(["same", "f32"]), act=act, gap=gap)
        return dict(op="affine", M=M, N=N, K=K, dtype=dtype, out=rng.choice(["same", "f32"]), act=act, residual=rng.random() < 0.5,
                    preact=act != "none" and rng.random() < 0.5, gap=gap)
    R, V = _log_int(rng, 1, 69120), _log_int(rng, 40, 131072)
    R = max(1, min(R, 69120 * 3000 // V))
    if rng.random() < 0.4:
        return dict(op="logprobs_grad", R=R, V=V, top=0, dtype=dtype, gap=gap)
    return dict(op="logprobs", R=R, V=V, top=rng.choice([0, 1, 3, 10, 20]), dtype=dtype, gap=gap)


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
    c = dict(case=case)
    if op in ("layer_norm", "layer_norm_grad"):
        R, H = case["R"], case["H"]
        c["x"] = s.rows(R, H, t, case["gap"], 1.5, 0.5 * s.normal(R, 1))
        c["weight"] = 1 + 0.2 * s.normal(H)
        if op == "layer_norm":
            c["bias"] = 0.1 * s.normal(H)
        else:
            c["dy"] = s.rows(R, H, t, case["gap"], 0.1)
            x = c["x"].float()                      # the statistics that the forward pass has handed over
            c["mean"] = x.mean(1)
            c["rstd"] = ((x - c["mean"][:, None]).square().mean(1) + EPS).rsqrt()
    elif op in ("affine", "affine_grad"):
        M, N, K = case["M"], case["N"], case["K"]
        c["x"] = s.rows(M, K, t, case["gap"])
        c["weight"] = s.rows(N, K, t, 0, K ** -0.5)
        if op == "affine":
            c["bias"] = 0.1 * s.normal(N)
            c["residual"] = s.rows(M, N, t if case["out"] == "same" else torch.float32, case["gap"]) if case["residual"] else None
        else:
            c["dy"] = s.rows(M, N, t if case["dy"] == "same" else torch.float32, case["gap"], 0.1)
            c["preact"] = s.rows(M, N, t, case["gap"]) if case["act"] != "none" else None
    else:
        R, V = case["R"], case["V"]
        x = 3 * s.normal(R, V + case["gap"])
        if R > 1:                                   # alternatives that are ruled out, and now and then a frame without any
            x.masked_fill_(s.uniform(R, V + case["gap"]) < 0.02, -math.inf)
            x.masked_fill_(s.uniform(R, 1) < 0.004, -math.inf)
        c["tokens"] = s.below(V, R)
        if R > 1:                                   # padded frames hold anything
            pad = s.uniform(R) < 0.1
            c["tokens"] = torch.where(pad, torch.full_like(c["tokens"], -1), c["tokens"])
            x.masked_fill_((pad & (s.uniform(R) < 0.5))[:, None], math.nan)
        c["logits"] = x.to(t)[:, :V]
        if op == "logprobs_grad":
            c["g_logprobs"], c["g_entropy"] = -1 - 0.1 * s.normal(R), -0.1 - 0.01 * s.normal(R)   # a sum over frames, as the objective is
            _, c["entropy"], c["logz"], _, _ = _logprobs(c["logits"], c["tokens"], 0)
    return c


# --------------------------------------------------------------------------- the plain forms

def _layer_norm(x, weight, bias):
    xf = x.float()
    mean = xf.mean(1)
    centred = xf - mean[:, None]
    rstd = (centred.square().mean(1) + EPS).rsqrt()
    return (centred * rstd[:, None] * weight + bias).to(x.dtype), mean, rstd


def _layer_norm_grad(dy, x, mean, rstd, weight):
    xh = (x.float() - mean[:, None]) * rstd[:, None]
    dyf = dy.float()
    g = dyf * weight
    dx = (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)) * rstd[:, None]
    return dx.to(x.dtype), (dyf * xh).sum(0), dyf.sum(0)


def _act(z, name):
    if name == "relu":
        return torch.where(z > 0, z, 0.0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_slope(z, name):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    s = 1 / (1 + torch.exp(-z))
    return s * (1 + z * (1 - s))


def _affine(x, weight, bias, act, residual, out_dtype, preact):
    z = x.float() @ weight.float().t() + bias
    y = _act(z, act)
    if residual is not None:
        y = y + residual.float()
    return (y.to(out_dtype), z.to(x.dtype)) if preact else y.to(out_dtype)


def _affine_grad(dy, x, weight, act, preact):
    dz = dy.float()
    if act != "none":
        dz = dz * _act_slope(preact.float(), act)
    return (dz @ weight.float()).to(x.dtype), (dz.t() @ x.float()).to(weight.dtype), dz.sum(0)


def _logprobs(logits, tokens, top):
    live = tokens >= 0
    x = torch.where(live[:, None], logits.float(), 0.0)
    m = x.max(1).values
    some = m > -math.inf
    d = x - torch.where(some, m, 0.0)[:, None]
    e = torch.exp(d)
    total = e.sum(1)
    logz = torch.where(some, m + torch.log(total), -math.inf)
    given = x.gather(1, tokens.clamp_min(0).long()[:, None])[:, 0]
    logprobs = torch.where(some, given - logz, -math.inf)
    entropy = torch.where(some, torch.log(total) - torch.where(e > 0, e * d, 0.0).sum(1) / total, 0.0)
    order = torch.sort(x, dim=1, descending=True, stable=True) if top else None
    ids = order.indices[:, :top].int() if top else torch.zeros((len(x), 0), dtype=torch.int32, device=x.device)
    best = order.values[:, :top] if top else torch.zeros((len(x), 0), device=x.device)
    best = torch.where(best > -math.inf, best - logz[:, None], -math.inf)
    zero = torch.zeros_like(logz)
    return (torch.where(live, logprobs, zero), torch.where(live, entropy, zero), torch.where(live, logz, zero),
            torch.where(live[:, None], ids, -1), torch.where(live[:, None], best, 0.0))


def _logprobs_grad(logits, tokens, logz, entropy, g_logprobs, g_entropy):
    live = (tokens >= 0) & (logz > -math.inf)
    logp = torch.where(live[:, None], logits.float() - logz[:, None], -math.inf)
    p = torch.exp(logp)
    d = -p * g_logprobs[:, None] - torch.where(p > 0, p * (logp + entropy[:, None]), 0.0) * g_entropy[:, None]
    at = tokens.clamp_min(0).long()[:, None]
    d.scatter_add_(1, at, torch.where(live, g_logprobs, 0.0)[:, None])
    return d.to(logits.dtype)


def run(c):
    case, op = c["case"], c["case"]["op"]
    if own:
        from paper_2112_00709_amd import layers as fl
        if op == "layer_norm":
            return fl.fb_layer_norm(c["x"], c["weight"], c["bias"], eps=EPS, want_stats=True)
        if op == "layer_norm_grad":
            return fl.fb_layer_norm_grad(c["dy"], c["x"], c["mean"], c["rstd"], c["weight"])
        if op == "affine":
            return fl.fb_affine(c["x"], c["weight"], c["bias"], activation=case["act"], residual=c["residual"],
                                out_dtype=None if case["out"] == "same" else torch.float32, want_preact=case["preact"])
        if op == "affine_grad":
            return fl.fb_affine_grad(c["dy"], c["x"], c["weight"], activation=case["act"], preact=c["preact"])
        if op == "logprobs":
            return fl.fb_token_logprobs(c["logits"], c["tokens"], top=case["top"])
        return fl.fb_token_logprobs_grad(c["logits"], c["tokens"], c["logz"], c["entropy"], c["g_logprobs"], c["g_entropy"])
    if op == "layer_norm":
        return _layer_norm(c["x"], c["weight"], c["bias"])
    if op == "layer_norm_grad":
        return _layer_norm_grad(c["dy"], c["x"], c["mean"], c["rstd"], c["weight"])
    if op == "affine":
        return _affine(c["x"], c["weight"], c["bias"], case["act"], c["residual"],
                       c["x"].dtype if case["out"] == "same" else torch.float32, case["preact"])
    if op == "affine_grad":
        return _affine_grad(c["dy"], c["x"], c["weight"], case["act"], c["preact"])
    if op == "logprobs":
        return _logprobs(c["logits"], c["tokens"], case["top"])
    return _logprobs_grad(c["logits"], c["tokens"], c["logz"], c["entropy"], c["g_logprobs"], c["g_entropy"])


# --------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    e, op = BYTES[case["dtype"]], case["op"]
    if op in ("layer_norm", "layer_norm_grad"):
        n, H = case["R"] * case["H"], case["H"]
        if op == "layer_norm":
            return {"bytes": 2 * n * e + 8 * H + 8 * case["R"], "flops": 8 * n}
        return {"bytes": 3 * n * e + 12 * H + 8 * case["R"], "flops": 14 * n}
    if op in ("affine", "affine_grad"):
        M, N, K = case["M"], case["N"], case["K"]
        if op == "affine":
            out = e if case["out"] == "same" else 4
            return {"bytes": (M * K + N * K) * e + 4 * N + M * N * (out * (2 if case["residual"] else 1) + (e if case["preact"] else 0)),
                    "flops": 2 * M * N * K}
        return {"bytes": 2 * (M * K + N * K) * e + 4 * N + M * N * ((e if case["dy"] == "same" else 4) + (e if case["act"] != "none" else 0)),
                "flops": 4 * M * N * K}
    R, V = case["R"], case["V"]
    if op == "logprobs":
        return {"bytes": R * (V * e + 4 + 12 + 8 * case["top"]), "flops": 6 * R * V}
    return {"bytes": R * (2 * V * e + 20), "flops": 8 * R * V}


# --------------------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    c, op, D = prepare(case, seed), case["op"], torch.float64
    if op == "layer_norm":
        var, mean = torch.var_mean(c["x"].to(D), dim=1, correction=0)
        rstd = 1 / torch.sqrt(var + EPS)
        return torch.addcmul(c["bias"].to(D), (c["x"].to(D) - mean.unsqueeze(1)) / torch.sqrt(var + EPS).unsqueeze(1), c["weight"].to(D)), mean, rstd
    if op == "layer_norm_grad":
        # through y_i = w_i (x_i - mean) / s: the Jacobian (I - 1 1'/H - xh xh'/H) / s applied to w * dy
        dy, s = c["dy"].to(D), 1 / c["rstd"].to(D).unsqueeze(1)
        u = (c["x"].to(D) - c["mean"].to(D).unsqueeze(1)) / s
        v = dy * c["weight"].to(D)
        dx = (v - v.sum(1, keepdim=True) / case["H"] - u * (u * v).sum(1, keepdim=True) / case["H"]) / s
        return dx, torch.sum(u * dy, 0), torch.sum(dy, 0)
    if op == "affine":
        z = torch.addmm(c["bias"].to(D), c["x"].to(D), c["weight"].to(D).t().contiguous())
        y = {"none": lambda: z.clone(), "relu": lambda: z.clamp_min(0), "gelu": lambda: z * torch.special.ndtr(z), "silu": lambda: z * torch.sigmoid(z)}[case["act"]]()
        if c["residual"] is not None:
            y += c["residual"].to(D)
        return (y, z) if case["preact"] else y
    if op == "affine_grad":
        g = c["dy"].to(D)
        if case["act"] != "none":
            z = c["preact"].to(D)
            if case["act"] == "relu":
                g = torch.where(z > 0, g, torch.zeros_like(g))
            elif case["act"] == "gelu":
                g = g * (torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
            else:
                g = g * (torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z))
        return torch.mm(g, c["weight"].to(D)), torch.mm(g.t().contiguous(), c["x"].to(D)), torch.sum(g, 0)
    pad = c["tokens"] < 0
    x = c["logits"].to(D).masked_fill(pad.unsqueeze(1), 0)
    if op == "logprobs":
        logz = torch.logsumexp(x, 1)
        dead = logz == -math.inf
        logp = (x - logz.unsqueeze(1)).masked_fill(dead.unsqueeze(1), -math.inf)
        entropy = torch.special.entr(torch.exp(logp)).sum(1)
        given = torch.take_along_dim(logp, c["tokens"].long().clamp_min(0).unsqueeze(1), 1).squeeze(1)
        best = torch.topk(logp, case["top"], dim=1).values if case["top"] else x.new_zeros((case["R"], 0))
        return (given.masked_fill(pad, 0), entropy.masked_fill(pad, 0), logz.masked_fill(pad, 0), None, best.masked_fill(pad.unsqueeze(1), 0))
    dead = pad | (c["logz"] == -math.inf)
    logp = (x - c["logz"].to(D).masked_fill(dead, 0).unsqueeze(1)).masked_fill(dead.unsqueeze(1), -math.inf)
    p = torch.exp(logp)
    hit = torch.zeros_like(p)
    hit.scatter_(1, c["tokens"].long().clamp_min(0).unsqueeze(1), 1.0)
    hit.masked_fill_(dead.unsqueeze(1), 0)
    inner = torch.xlogy(p, p) + p * c["entropy"].to(D).unsqueeze(1)
    return (hit - p) * c["g_logprobs"].to(D).unsqueeze(1) - inner * c["g_entropy"].to(D).unsqueeze(1)
