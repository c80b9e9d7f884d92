"""From hidden states to a partition: trains a small residual encoder as an auto-encoder, encodes a data set with it and
partitions the features (the paper takes its features from the bottleneck of such an auto-encoder).

    python examples/encode_and_partition.py [--samples 20000] [--width 512] [--inner 1408] [--features 128] [--steps 60] [--bits 8]

A layer is  norm(x + r) -> gated block -> product with the residual in its epilogue; the head is a norm and a product down to
the features, the decoder one product back.  Training runs the operators' gradients in bf16 under Adam;
encoding runs the same layers forward, with --bits 8 on 8-bit weights and activations with block scales.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2211_00839_amd as rcd  # noqa: E402

EPS = 1e-6


def make_hidden_states(samples, width, classes, seed):
    """Stand-in for a text model's hidden states: per class a low-dimensional cloud of its own in `width` dimensions."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    labels = torch.randint(0, classes, (samples,), generator=gen, device="cuda", dtype=torch.int32)
    basis = torch.randn(classes, 16, width, generator=gen, device="cuda") / 4
    centre = torch.randn(classes, width, generator=gen, device="cuda")
    x = torch.empty(samples, width, device="cuda")
    for c in range(classes):
        at = (labels == c).nonzero().flatten()
        x[at] = centre[c] + torch.randn(len(at), 16, generator=gen, device="cuda") @ basis[c]
    return (x + 0.1 * torch.randn(samples, width, generator=gen, device="cuda")).bfloat16(), labels


class Encoder:
    def __init__(self, width, inner, features, layers, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def weight(rows, cols, gain=1.0):
            return (torch.randn(rows, cols, generator=gen, device="cuda") * gain * cols ** -0.5).bfloat16()

        self.p = {}
        for i in range(layers):
            self.p["scale%d" % i] = torch.ones(width, dtype=torch.bfloat16, device="cuda")
            self.p["gate%d" % i], self.p["up%d" % i] = weight(inner, width), weight(inner, width)
            self.p["down%d" % i] = weight(width, inner, 0.5)
        self.p["scale"] = torch.ones(width, dtype=torch.bfloat16, device="cuda")
        self.p["head"], self.p["head_bias"] = weight(features, width), torch.zeros(features, dtype=torch.bfloat16, device="cuda")
        self.p["back"], self.p["back_bias"] = weight(width, features), torch.zeros(width, dtype=torch.bfloat16, device="cuda")
        self.layers = layers
        self.master = {k: v.float() for k, v in self.p.items()}
        self.moments = {k: (torch.zeros_like(v), torch.zeros_like(v)) for k, v in self.master.items()}
        self.steps = 0

    def loss_and_gradients(self, x):
        """Mean squared error of the reconstruction, and the gradient of every parameter."""
        p, kept, grad = self.p, [], {}
        r = x
        for i in range(self.layers):
            n = rcd.rms_norm(r, p["scale%d" % i], EPS, want_rstd=True)
            h, saved = rcd.gated_linear(n.y, p["gate%d" % i], p["up%d" % i], want_saved=True)
            out = rcd.linear(h, p["down%d" % i], residual=r)
            kept.append((r, n, h, saved))
            r = out
        n = rcd.rms_norm(r, p["scale"], EPS, want_rstd=True)
        features = rcd.linear(n.y, p["head"], p["head_bias"])
        made = rcd.linear(features, p["back"], p["back_bias"])
        off = made.float() - x.float()
        loss = off.square().mean()
        d = (off * (2.0 / off.shape[0])).bfloat16()            # (a sum over the width, a mean over the samples)
        df, grad["back"], grad["back_bias"] = rcd.linear_backward(d, features, p["back"])
        dn, grad["head"], grad["head_bias"] = rcd.linear_backward(df, n.y, p["head"])
        dr, grad["scale"] = rcd.rms_norm_backward(dn, r, n.rstd, p["scale"])
        for i in reversed(range(self.layers)):
            r, n, h, saved = kept[i]
            dh, grad["down%d" % i], _ = rcd.linear_backward(dr, h, p["down%d" % i], want_dbias=False)
            dn, grad["gate%d" % i], grad["up%d" % i] = rcd.gated_linear_backward(dh, n.y, p["gate%d" % i], p["up%d" % i], saved)
            dr, grad["scale%d" % i] = rcd.rms_norm_backward(dn, r, n.rstd, p["scale%d" % i], dsum=dr)
        return loss, grad

    def step(self, grad, rate):
        """Adam (0.9, 0.999) on fp32 copies of the weights."""
        self.steps += 1
        for k, g in grad.items():
            first, second = self.moments[k]
            g = g.float()
            first.lerp_(g, 0.1)
            second.lerp_(g * g, 0.001)
            size = (second / (1 - 0.999 ** self.steps)).sqrt() + 1e-8
            self.master[k].sub_(rate / (1 - 0.9 ** self.steps) * first / size)
            self.p[k].copy_(self.master[k])

    def encode(self, x):
        """Features of the rows of x, bf16 throughout."""
        p, r = self.p, x
        for i in range(self.layers):
            h = rcd.gated_linear(rcd.rms_norm(r, p["scale%d" % i], EPS).y, p["gate%d" % i], p["up%d" % i])
            r = rcd.linear(h, p["down%d" % i], residual=r)
        return rcd.linear(rcd.rms_norm(r, p["scale"], EPS).y, p["head"], p["head_bias"])

    def quantize(self):
        """The weights in 8 bits with block scales, laid out once."""
        self.q = {k: rcd.quantize_mxfp8(v) for k, v in self.p.items() if v.dim() == 2}

    def encode_8_bits(self, x):
        """The same on 8-bit weights: every norm hands its output on in 8 bits, and so does the gated block's through the quantizer."""
        p, q, r = self.p, self.q, x
        for i in range(self.layers):
            n = rcd.rms_norm(r, p["scale%d" % i], EPS, quantize=True)
            (gate, gate_scale), (up, up_scale), (down, down_scale) = (q[k + str(i)] for k in ("gate", "up", "down"))
            h, h_scale = rcd.quantize_mxfp8(rcd.gated_linear(n.y, gate, up, a_scale=n.scale, gate_scale=gate_scale, up_scale=up_scale))
            r = rcd.linear(h, down, residual=r, a_scale=h_scale, w_scale=down_scale)
        n = rcd.rms_norm(r, p["scale"], EPS, quantize=True)
        head, head_scale = q["head"]
        return rcd.linear(n.y, head, p["head_bias"], a_scale=n.scale, w_scale=head_scale)


def run(samples=20000, width=512, inner=1408, features=128, classes=10, layers=2, steps=60, batch=2048, bits=8, rate=0.002, seed=0, say=print):
    x, labels = make_hidden_states(samples, width, classes, seed)
    model = Encoder(width, inner, features, layers, seed + 1)
    pick = torch.Generator(device="cuda").manual_seed(seed + 2)
    losses = []
    for t in range(steps):
        at = torch.randint(0, samples, (min(batch, samples),), generator=pick, device="cuda")
        loss, grad = model.loss_and_gradients(x[at])
        model.step(grad, rate)
        losses.append(loss)
        if t % 20 == 0 or t == steps - 1:
            say("step %3d: reconstruction error %.4f" % (t, loss.item()))
    plain = model.encode(x)
    made = plain
    if bits == 8:
        model.quantize()
        made = model.encode_8_bits(x)
        say("8-bit features are %.2f %% off the bf16 ones" % (100 * ((made.float() - plain.float()).norm() / plain.float().norm()).item()))
    sigma = rcd.bandwidth(made[: min(samples, 4000)].contiguous())
    r = np.array([1, 1, 2, 4], dtype=np.int32)
    most = int(torch.bincount(labels, minlength=classes).max())
    _, room = rcd.dataset_workspace_bytes(samples, classes, most, len(r), rcd.MODE_INCREMENTAL)
    workspace = torch.empty(room, dtype=torch.uint8, device="cuda")
    assign, order, obj = rcd.partition_dataset(made, labels, classes, r, float(sigma) ** 2, rcd.MODE_AUTO, workspace)
    counts = torch.bincount(assign, minlength=len(r)).tolist()
    say("bandwidth %.3f; %d workers of capacities %s got %s samples" % (sigma, len(r), r.tolist(), counts))
    return {"losses": [float(v) for v in losses], "features": made, "plain": plain, "labels": labels, "assign": assign, "objective": obj, "counts": counts}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("samples", 20000), ("width", 512), ("inner", 1408), ("features", 128), ("classes", 10), ("layers", 2), ("steps", 60), ("bits", 8)):
        ap.add_argument("--" + name, type=int, default=value)
    run(**vars(ap.parse_args()))
