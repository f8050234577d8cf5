"""A small network that learns from decoded batches: patches of every image as rows, blocks of norm and two linear layers, class scores.

The consumer of the decode (Sec. III-B hands the decoded batch to a backbone): a batch of image ids is decoded on the GPU, cut into
patches and learned from without leaving it.  Every dense operator is one of rinr_nn's; what is kept between the forward and the backward
pass are the sums that norms were taken of and, in 8 bits, what the first layers of the blocks read and what their activations are taken of.

`python -m paper_2306_16699_amd.backbone` trains one on a synthetic store whose images' classes differ in colour.
"""
from __future__ import annotations

import argparse
import math
import time

import numpy as np
import torch

from . import rinr, rinr_nn as nn, synth


class Backbone:
    """h = patches w_in' + b_in; per block h += w2 gelu(w1 norm(h) + b1) + b2; scores = w_out mean(norm(h)) + b_out.

    Parameters are kept in 32 bits (`params`); products take the weights as `dtype`."""

    def __init__(self, patch: int, width: int, hidden: int, blocks: int, classes: int, dtype=torch.bfloat16, device="cuda:0", seed: int = 0):
        g = torch.Generator().manual_seed(seed)

        def weights(n_out, n_in, scale=1.0):
            return (torch.randn((n_out, n_in), generator=g) * (scale / math.sqrt(n_in))).to(device)

        self.patch, self.blocks, self.dtype = patch, blocks, dtype
        p = {"w_in": weights(width, 3 * patch * patch), "b_in": torch.zeros(width, device=device)}
        for k in range(blocks):
            p[f"gain{k}"] = torch.ones(width, device=device)
            p[f"w1_{k}"], p[f"b1_{k}"] = weights(hidden, width), torch.zeros(hidden, device=device)
            p[f"w2_{k}"], p[f"b2_{k}"] = weights(width, hidden, 1.0 / math.sqrt(blocks)), torch.zeros(width, device=device)
        p["gain_out"] = torch.ones(width, device=device)
        p["w_out"], p["b_out"] = weights(classes, width), torch.zeros(classes, device=device)
        self.params = p
        self._round()

    def _round(self):
        self.weights = {k: v.to(self.dtype) for k, v in self.params.items() if v.dim() == 2}

    def patches(self, images):
        """[n, 3, H, W] -> [n * patches, 3 * patch * patch] of the products' type, a patch's values channel by channel."""
        n, c, H, W = images.shape
        s = self.patch
        if H % s or W % s:
            raise rinr.RinrError(rinr.E_ARG, f"images of {H} x {W} in patches of {s} x {s}")
        return images.view(n, c, H // s, s, W // s, s).permute(0, 2, 4, 1, 3, 5).to(self.dtype).reshape(-1, c * s * s)

    def forward(self, images, keep: bool = False):
        """Class scores [n, classes] in 32 bits; with `keep` also what backward() needs."""
        p, w, n = self.params, self.weights, images.shape[0]
        x = self.patches(images)
        h = nn.linear(x, w["w_in"], p["b_in"])
        tape = [x]
        for k in range(self.blocks):
            y, _ = nn.rms_norm(h, p[f"gain{k}"], packed=True)
            a, z = nn.linear(y, w[f"w1_{k}"], p[f"b1_{k}"], act="gelu", keep_z="packed")
            tape.append((h, y, z))
            h = nn.linear(a, w[f"w2_{k}"], p[f"b2_{k}"], residual=h)
        y, _ = nn.rms_norm(h, p["gain_out"])
        mean = y.view(n, -1, y.shape[1]).float().mean(1).to(self.dtype)
        scores = nn.linear(mean, w["w_out"], p["b_out"]).float()
        return (scores, tape + [h, mean]) if keep else scores

    def backward(self, tape, dscores):
        """Gradients of the parameters, given those of the scores."""
        p, w, g = self.params, self.weights, {}
        x, *kept, h, mean = tape
        dmean, g["w_out"], g["b_out"] = nn.linear_backward(dscores.to(self.dtype), mean, w["w_out"])
        per_image = h.shape[0] // mean.shape[0]
        dy = (dmean.float() / per_image).to(self.dtype).repeat_interleave(per_image, dim=0)
        dh, g["gain_out"] = nn.rms_norm_backward(dy, h, p["gain_out"])
        for k in reversed(range(self.blocks)):
            h, y, z = kept[k]
            dz, g[f"w2_{k}"], g[f"b2_{k}"] = nn.linear_backward(dh, z, w[f"w2_{k}"], x_act="gelu")
            dy, g[f"w1_{k}"], g[f"b1_{k}"] = nn.linear_backward(dz, y, w[f"w1_{k}"])
            dh, g[f"gain{k}"] = nn.rms_norm_backward(dy, h, p[f"gain{k}"], dres=dh)
        _, g["w_in"], g["b_in"] = nn.linear_backward(dh, x, w["w_in"], need_dx=False)
        return g

    def step(self, images, labels, lr: float):
        """One step of gradient descent on the mean cross entropy; returns it (a device scalar)."""
        scores, tape = self.forward(images, keep=True)
        logp = scores - scores.logsumexp(1, keepdim=True)
        loss = -logp.gather(1, labels[:, None]).mean()
        d = logp.exp()
        d.scatter_add_(1, labels[:, None], torch.full_like(d[:, :1], -1.0))
        for k, g in self.backward(tape, d / labels.numel()).items():
            self.params[k].sub_(g.float(), alpha=lr)
        self._round()
        return loss


def colour_store(n_images: int, classes: int, seed: int = 0):
    """A store of synthetic models and their labels: a class's images are tinted alike."""
    labels = np.arange(n_images) % classes
    models = synth.make_models(seed, np.arange(n_images), 24, 3, [0, 8, 8, 0], 0.8)
    tint = np.random.default_rng(seed).uniform(0.25, 0.75, (classes, 3)).astype(np.float32)
    for m, c in zip(models, labels):
        m.layers[-1].bias = m.layers[-1].bias + tint[c]
    return rinr.Store(rinr.pack(models)), torch.from_numpy(labels).to("cuda:0")


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--images", type=int, default=512)
    ap.add_argument("--size", type=int, default=224)
    ap.add_argument("--patch", type=int, default=14)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--hidden", type=int, default=2048)
    ap.add_argument("--blocks", type=int, default=4)
    ap.add_argument("--classes", type=int, default=10)
    ap.add_argument("--batch", type=int, default=64)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--lr", type=float, default=0.01)
    a = ap.parse_args()
    store, labels = colour_store(a.images, a.classes)
    net = Backbone(a.patch, a.width, a.hidden, a.blocks, a.classes)
    g = torch.Generator().manual_seed(1)
    t = 0.0
    for step in range(a.steps):
        ids = torch.randint(0, a.images, (a.batch,), generator=g).to("cuda:0")
        loss = net.step(store.decode_batch(ids, a.size, a.size), labels[ids], a.lr)
        if step % 10 == 0 or step == a.steps - 1:
            value = loss.item()
            if step == 0:                                              # without what the first step sets up
                t = time.perf_counter()
            took = f", {(time.perf_counter() - t) * 1e3 / step:.2f} ms a step" if step else ""
            print(f"step {step}: cross entropy {value:.4f}{took}", flush=True)


if __name__ == "__main__":
    main()
