"""The last layers of an acoustic network trained with the LF-MMI objective, on synthetic frames.

    python examples/network_head.py [--dtype bfloat16] [--steps 20]

Hidden frames go through layer norm, a hidden layer with a skip connection, layer norm and the output layer, whose
single-precision outputs are the objective's pseudo-log-likelihoods.  Beside LF-MMI, the frames' log probabilities on the best
path through the numerator graphs are raised (cross-entropy on an alignment) and their entropy is kept up a little.  Then the
trained layers serve one frame at a time, with the best alternatives.  Everything but the parameters' update runs in this
library's kernels.
"""
from __future__ import annotations

import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


class Head:
    """hidden [..., H] -> emissions float32 [..., D].  Parameters are kept in single precision; products run in ``dtype``."""

    def __init__(self, H, F, D, dtype, device="cuda", seed=0):
        import torch
        gen = torch.Generator().manual_seed(seed)

        def normal(n, k):
            return (torch.randn((n, k), generator=gen) * k ** -0.5).to(device).requires_grad_(True)

        def full(n, v):
            return torch.full((n,), float(v), device=device, requires_grad=True)

        self.dtype = dtype
        self.params = dict(norm0_w=full(H, 1), norm0_b=full(H, 0), hidden_w=normal(F, H), hidden_b=full(F, 0), back_w=normal(H, F), back_b=full(H, 0),
                           norm1_w=full(H, 1), norm1_b=full(H, 0), out_w=normal(D, H), out_b=full(D, 0))

    def __call__(self, hidden):
        import torch

        from paper_2112_00709_amd import autograd as fa
        p, t = self.params, self.dtype
        x = fa.layer_norm(hidden, p["norm0_w"], p["norm0_b"])
        x = fa.affine(x, p["hidden_w"].to(t), p["hidden_b"], activation="gelu")
        x = fa.affine(x, p["back_w"].to(t), p["back_b"], residual=hidden)
        x = fa.layer_norm(x, p["norm1_w"], p["norm1_b"])
        return fa.affine(x, p["out_w"].to(t), p["out_b"], out_dtype=torch.float32)


def alignment(num, num_pdf, emis, lengths):
    """The pdf of every frame on the best path through the utterance's numerator graph, -1 on padded frames (int32 [B, N])."""
    import torch

    import paper_2112_00709_amd as fb
    _, path = fb.fb_viterbi(num, emis.detach(), lengths)
    return torch.where(path >= 0, num_pdf[path.clamp_min(0).long()], -1).to(torch.int32)


def train(head, hidden, w, den, num, steps, rate=0.2, ce=0.5, entropy=0.05):
    """Gradient ascent on LF-MMI per frame + ce * frame log probability + entropy * frame entropy; -> the three, a step each."""
    import torch

    from paper_2112_00709_amd import autograd as fa
    lengths = torch.from_numpy(w.lengths).cuda()
    frames = int(w.lengths.sum())
    num_pdf = torch.from_numpy(w.num.pdf).cuda()
    log = []
    for _ in range(steps):
        emis = head(hidden)
        mmi, _, _ = fa.lfmmi_loss(emis, lengths, den, num)
        logprobs, ent, _, _, _ = fa.token_logprobs(emis, alignment(num, num_pdf, emis, lengths))
        terms = mmi.float().sum() / frames, logprobs.sum() / frames, ent.sum() / frames
        (terms[0] + ce * terms[1] + entropy * terms[2]).backward()
        with torch.no_grad():
            for p in head.params.values():
                p += rate * p.grad
                p.grad = None
        log.append(tuple(float(x.detach()) for x in terms))
    return log


def serve(head, hidden, top=5):
    """One frame [H] after the other: -> (best pdfs [n, top], their log probabilities, entropies)."""
    import torch

    from paper_2112_00709_amd import layers as fl
    ids, best, ents = [], [], []
    with torch.no_grad():
        for frame in hidden:
            emis = head(frame[None])
            token = torch.zeros((1,), dtype=torch.int32, device=emis.device)
            _, ent, _, i, b = fl.fb_token_logprobs(emis, token, top=top)
            ids.append(i)
            best.append(b)
            ents.append(ent)
    return torch.cat(ids), torch.cat(best), torch.cat(ents)


def setup(K=1200, B=12, D=96, H=192, dtype="float32"):
    """Graphs and lengths of a small LF-MMI workload, and hidden frames that know something of the reference pdfs."""
    import torch

    import paper_2112_00709_amd as fb
    import workloads as wl
    w = wl.config5(K=K, B=B, Lmin=4, Lmax=12, D=D)
    den, num = fb.graph_from(w.den, w.D), fb.graph_from(w.num, w.D)
    gen = torch.Generator().manual_seed(1)
    emis = torch.from_numpy(w.emis).cuda()
    mix = (torch.randn((w.D, H), generator=gen) * w.D ** -0.5).cuda()
    noise = torch.randn((w.B, w.N, H), generator=gen).cuda()
    hidden = (torch.nan_to_num(emis) @ mix * 0.5 + 0.5 * noise).to(getattr(torch, dtype))
    return w, den, num, hidden


def main(argv=None):
    import torch
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--dtype", choices=("float32", "bfloat16", "float16"), default="bfloat16")
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args(argv)
    w, den, num, hidden = setup(dtype=a.dtype)
    head = Head(hidden.shape[-1], 384, w.D, getattr(torch, a.dtype))
    log = train(head, hidden, w, den, num, a.steps)
    for i, (mmi, ce, ent) in enumerate(log):
        print(f"step {i}: LF-MMI {mmi:.4f}  log probability on the alignment {ce:.4f}  entropy {ent:.4f}", flush=True)
    ids, best, ents = serve(head, hidden[0, :4])
    for i in range(len(ids)):
        print(f"frame {i}: entropy {float(ents[i]):.3f}, best", ", ".join(f"{int(j)} ({float(b):.2f})" for j, b in zip(ids[i], best[i])), flush=True)
    for g in (den, num):
        g.destroy()
    return log


if __name__ == "__main__":
    main()
