"""Fitting a length predictor to observed output lengths (the paper's post-execution profiling feeds
them back into the predictor).

A step takes the batch's features through the layers (activations kept), reads the log probability of
every stage's observed length bin, takes the gradient of their mean back through the layers, clips it
by its global norm and moves float32 master weights by it (momentum), from which the predictor's own
weights are rounded; a batch whose gradient's norm is not finite moves nothing. All but the update runs in the
library's kernels, in the buffers a ``Fit`` holds; nothing in a step synchronises. The weights are the ones ``predict`` takes.

    python -m paper_2606_12950_amd.fit --workload c1 --stages 65536 --steps 50
"""
from __future__ import annotations

import argparse
import math
from typing import List, Optional, Sequence, Tuple

import torch

from . import _native, _train
from ._train import LayerGrad, Logprobs, clip_gradients, layer, layer_grad, logprobs, logprobs_grad


def bins_of(length: torch.Tensor, bin_centre: torch.Tensor) -> torch.Tensor:
    """int32 bin of every observed length: the one with the nearest centre (ascending centres, the lower of
    two as near); a length that is not finite (none observed) is -1."""
    middle = (bin_centre[1:] + bin_centre[:-1]) / 2
    at = torch.bucketize(length.to(middle.dtype), middle).to(torch.int32)
    return torch.where(torch.isfinite(length), at, -1)


class Fit:
    """A predictor being fitted: its weights, their float32 masters, and the buffers of batches of ``n`` stages.

    ``weights`` [out][in] (float32 or bfloat16) and ``biases`` (float32) are updated in place.
    ``entropy_bonus`` adds that much times the mean entropy to what is maximised."""

    def __init__(self, weights: Sequence[torch.Tensor], biases: Sequence[torch.Tensor], n: int,
                 entropy_bonus: float = 0.0):
        _native.make_predictor(weights, biases, None)      # the same checks as predict's
        self.weights, self.biases, self.n = list(weights), list(biases), n
        dt, dev = weights[0].dtype, weights[0].device
        widths = [weights[0].shape[1]] + [w.shape[0] for w in weights]
        f = dict(dtype=torch.float32, device=dev)
        # masters, gradients and velocities each end to end, weights first (16-byte aligned: widths are multiples of 16), so
        # that an update takes few launches
        L, size = len(weights), sum(t.numel() for t in (*weights, *biases))
        views = lambda flat, like: [v.view(t.shape) for v, t in zip(flat.split([t.numel() for t in like]), like)]
        self._master = torch.cat([w.reshape(-1).float() for w in weights])
        self._gradient, self._velocity = torch.zeros(size, **f), torch.zeros(size, **f)
        self.masters, self.velocity = views(self._master, weights), views(self._velocity, [*weights, *biases])
        gradients = views(self._gradient, [*weights, *biases])
        self.g_weights, self.g_biases = gradients[:L], gradients[L:]
        self.hidden = [torch.empty(n, w, dtype=dt, device=dev) for w in widths[1:]]      # the last: logits
        self.g_z = [torch.empty_like(h) for h in self.hidden]
        self.out = Logprobs(torch.empty(n, **f), torch.empty(n, **f), torch.empty(n, 0, dtype=torch.int32, device=dev),
                            torch.empty(n, 0, **f), torch.empty(n, 2, **f))
        self.entropy_bonus = entropy_bonus
        self.g_entropy = torch.full((n,), entropy_bonus / max(n, 1), **f) if entropy_bonus else None
        self.norm = torch.empty(1, **f)
        lib, code = _train.load(), _train._DTYPE[dt]
        need = [lib.maestro_layer_grad_workspace(n, i, o, code) for i, o in zip(widths[:-1], widths[1:])]
        need += [lib.maestro_logprobs_workspace(n, widths[-1], 0, code),
                 lib.maestro_clip_gradients_workspace(2 * len(weights)), 16]
        self.workspace = torch.empty(max(need), dtype=torch.uint8, device=dev)

    def score(self, x: torch.Tensor, bins: torch.Tensor) -> Logprobs:
        """The layers forward and the observed bins' log probabilities (0 where none was observed), in the Fit's buffers:
        the next call writes them again."""
        h = x
        for l, (w, b) in enumerate(zip(self.weights, self.biases)):
            h = layer(h, w, b, relu=l + 1 < len(self.weights), out=self.hidden[l])
        return logprobs(h, bins, out=self.out, workspace=self.workspace)

    def _given(self, bins: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
        """Which stages' bins were observed, and how many (1 where none)."""
        given = (bins >= 0) & (bins < self.hidden[-1].shape[1])
        return given, given.sum().clamp_min(1)

    def gradients(self, x: torch.Tensor, bins: torch.Tensor) -> Tuple[List[torch.Tensor], List[torch.Tensor]]:
        """Gradients of minus the mean log probability of the observed bins (less the entropy bonus), of
        weights and biases, after ``score``, in the Fit's buffers: the next call writes them again. Features
        have to be finite, also those of stages without an observed bin."""
        return self._gradients(x, bins, *self._given(bins))

    def _gradients(self, x, bins, given, count):
        g = given.float() / -count
        ge = None if self.g_entropy is None else -self.g_entropy
        logprobs_grad(self.hidden[-1], bins, self.out.stats, self.out.entropy, g, ge, out=self.g_z[-1])
        for l in reversed(range(len(self.weights))):
            below = l > 0
            layer_grad(self.hidden[l - 1] if below else x, self.weights[l], self.g_z[l], relu_input=below, want_x=below,
                       out=LayerGrad(self.g_z[l - 1] if below else None, self.g_weights[l], self.g_biases[l]),
                       workspace=self.workspace)
        return self.g_weights, self.g_biases

    def step(self, x: torch.Tensor, bins: torch.Tensor, rate: float, max_norm: float = 1.0,
             momentum: float = 0.9) -> Tuple[torch.Tensor, torch.Tensor]:
        """One update; where the gradient's norm is not finite, weights, biases and velocities stay as they are. Returns
        the mean log probability before it and the norm before clipping, on the device, in tensors of their own (the
        ones that ``score`` and ``gradients`` return are the Fit's buffers, which the next call writes). Stages without
        an observed bin take no part, whatever their features hold (with an entropy bonus they take part in that, and
        their features have to be finite)."""
        width = self.weights[0].shape[1]
        _native._shape(_native._dev(x, "x", self.weights[0].dtype), "x", (self.n, width))
        _native._shape(_native._dev(bins, "bins", torch.int32), "bins", (self.n,))
        given, count = self._given(bins)
        if not self.entropy_bonus:
            x = torch.where(given[:, None], x, 0.0)        # 0 times a NaN would be one in the weights' gradient
        out = self.score(x, bins)
        mean = out.logprob.sum() / count
        self._gradients(x, bins, given, count)
        grads = [*self.g_weights, *self.g_biases]
        clip_gradients(grads, max_norm, norm=self.norm, workspace=self.workspace)
        finite, v = self.norm < math.inf, self._velocity * momentum       # a NaN is not less
        v.add_(self._gradient)
        by, at = torch.where(finite, v, 0.0), self._master.numel()
        torch.where(finite, v, self._velocity, out=self._velocity)
        self._master.add_(by[:at], alpha=-rate)
        for b in self.biases:
            b.add_(by[at:at + b.numel()], alpha=-rate)
            at += b.numel()
        for w, p in zip(self.weights, self.masters):
            w.copy_(p)
        return mean, self.norm.clone()


def main(argv: Optional[Sequence[str]] = None) -> dict:
    from . import pipeline
    from . import workload as W

    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--workload", default="c1", choices=sorted(W.SPECS))
    ap.add_argument("--stages", type=int, default=None, help="stages of the batch (default: the workload's)")
    ap.add_argument("--steps", type=int, default=50)
    ap.add_argument("--rate", type=float, default=0.2)
    ap.add_argument("--max-norm", type=float, default=1.0)
    a = ap.parse_args(argv)
    if a.steps < 1:
        ap.error("--steps must be at least 1")
    if W.SPECS[a.workload].n_workflows:
        ap.error("a workload of single stages is needed")
    wl = W.workload(a.workload, **({} if a.stages is None else dict(n_stages=a.stages)))
    b = pipeline.to_device(wl)
    # lengths that depend on the features: a fixed direction of them, spread over the bins
    g = torch.Generator(device=b.x.device)
    g.manual_seed(0)
    d = torch.randn(b.x.shape[1], generator=g, device=b.x.device)
    t = torch.sigmoid(b.x.float() @ (d / d.norm()) * 1.5)
    length = b.bin_centre[0] + t * (b.bin_centre[-1] - b.bin_centre[0])
    bins = bins_of(length, b.bin_centre)
    fit = Fit(b.weights, b.biases, b.n)

    def error() -> float:
        pred, _ = _native.predict(b.x, b.weights, b.biases, b.bin_centre, b.prompt_len, b.model_id, b.kv_bytes_per_token)
        return float((pred - length).abs().mean())

    before, first = error(), None
    for s in range(a.steps):
        mean, norm = fit.step(b.x, bins, a.rate, a.max_norm)
        first = float(mean) if first is None else first
        if s % 10 == 9 or s == a.steps - 1:
            print(f"step {s + 1}: mean log probability {float(mean):.4f}, gradient norm {float(norm):.4f}", flush=True)
    result = dict(stages=b.n, first=first, last=float(fit.score(b.x, bins).logprob.mean()), error_before=before,
                  error_after=error())
    print("mean log probability {first:.4f} -> {last:.4f}; predicted length off by {error_before:.1f} -> "
          "{error_after:.1f} tokens over {stages} stages".format(**result), flush=True)
    return result


if __name__ == "__main__":
    main()
