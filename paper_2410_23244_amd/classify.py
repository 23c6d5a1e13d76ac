"""Categorical outcomes: one probit forest per class, its scores turned into
calibrated probabilities.

The sampler answers with a number or, by the probit model, with a yes or no.
:class:`Classifier` fits one probit forest per class (that class or any other),
all with the same number of chains, and so gets a score per class and
observation: the posterior mean of that forest's f.  :class:`Calibration`
learns, on observations held out from the forests, how scores become log
probabilities, by minimising the log loss: :func:`ops.logprob` gives the loss
with its gradient, :class:`ops.AdamW` steps all chains' weights at once, and
:func:`ops.logprob` then answers with log probabilities, entropies and the best
alternatives.
"""
from __future__ import annotations

import math
from statistics import NormalDist

import numpy as np

from . import ops
from .bart import (BART_EDEVICE, BART_EINVAL, BART_GRID_QUANTILE, Bart, BartError, bart_bin,
                   bart_cutpoints)


class Calibration:
    """Per chain, logits = s + s D^T + b from scores s [chains, n, classes]
    (float32): D and b start at 0, so that logits start as the scores; decay
    pulls D back there.

    fit minimises -mean log p(label) (rows with a negative label do not
    count) by full-batch AdamW over the 2 x chains tensors."""

    def __init__(self, n_class: int, chains: int = 1, lr: float = 3e-2,
                 weight_decay: float = 1e-3, state_bits: int = 32, device: str = "cuda"):
        import torch

        if n_class < 2 or chains < 1:
            raise BartError(BART_EINVAL, "a calibration needs 2 classes and 1 chain at least")
        self.torch, self.n_class, self.chains = torch, n_class, chains
        dev = torch.device(device, torch.cuda.current_device()) if device == "cuda" else device

        def zeros(*shape):
            return [torch.zeros(shape, device=dev) for _ in range(chains)]

        self.D, self.b = zeros(n_class, n_class), zeros(n_class)
        self._dD, self._db = zeros(n_class, n_class), zeros(n_class)
        self.opt = ops.AdamW(self.D + self.b, self._dD + self._db, lr=lr, state_bits=state_bits,
                             weight_decay=[weight_decay] * chains + [0.0] * chains)
        self._held = ops.Held(self.D + self.b + self._dD + self._db, self.opt.device)

    def _check(self, scores):
        if scores.dim() != 3 or scores.shape[0] != self.chains or \
                scores.shape[2] != self.n_class or scores.dtype != self.torch.float32:
            raise BartError(BART_EINVAL, f"scores must be float32 [{self.chains}, rows, "
                                         f"{self.n_class}]")
        dev = self.opt.device
        self._held.use(dev, self.torch.cuda.current_stream(dev).cuda_stream)

    def logits(self, scores, chain: int):
        return self.torch.addmm(scores[chain], scores[chain], self.D[chain].t()).add_(
            self.b[chain])

    def fit(self, scores, labels, steps: int = 200):
        """Returns the log loss before each step, [steps, chains] on the device."""
        torch = self.torch
        self._check(scores)
        n = (labels >= 0).sum().clamp(min=1)
        weight = (-1.0 / n).float()                     # of log p, the same for all rows
        losses = torch.empty((steps, self.chains), device=scores.device)
        for t in range(steps):
            for c in range(self.chains):
                z = self.logits(scores, c)
                r = ops.logprob(z, labels, grad_logp=weight, grad_out=z)
                torch.mm(r.grad.t(), scores[c], out=self._dD[c])
                torch.sum(r.grad, 0, out=self._db[c])
                losses[t, c] = r.logp.sum() * weight
            self.opt.step()
        return losses

    def answer(self, scores, labels=None, k: int = 1) -> ops.LogProb:
        """Log probabilities of given labels, entropies and the best k classes, from
        the chains' mean logits."""
        self._check(scores)
        z = self.logits(scores, 0)
        for c in range(1, self.chains):
            z += self.logits(scores, c)
        return ops.logprob(z.div_(self.chains), labels, k=k, entropy=True)


class Classifier:
    """Classification of X (f32 [n][p], one row per observation) into the
    classes 0 ... n_class - 1 of y.

    fit holds out a share of the observations, runs n_class probit forests of
    nchain chains on the others (bins and cuts as Regressor's), scores the held
    out and the test points over the kept sweeps and calibrates on the former.
    Afterwards: answer(y_test, k) over the test points; scores, float32
    [nchain, n_test, n_class] on the device; losses of the calibration."""

    def __init__(self, ntree: int = 200, max_depth: int = 6, K: int = 255,
                 grid: int = BART_GRID_QUANTILE, nchain: int = 1, seed: int = 0,
                 holdout: float = 0.25, calibration_steps: int = 200):
        self.ntree, self.max_depth, self.K, self.grid = ntree, max_depth, K, grid
        self.nchain, self.seed, self.holdout = nchain, seed, holdout
        self.calibration_steps = calibration_steps

    def fit(self, X, y, X_test, n_burn: int = 100, n_keep: int = 200):
        import torch

        y = np.asarray(y)
        if y.ndim != 1 or y.size < 2 or not np.issubdtype(y.dtype, np.integer) or y.min() < 0:
            raise BartError(BART_EINVAL, "y must be classes 0, 1, ... of at least 2 observations")
        if not 0.0 < self.holdout < 1.0:
            raise BartError(BART_EINVAL, "holdout must be between 0 and 1")
        X, X_test = np.asarray(X, dtype=np.float32), np.asarray(X_test, dtype=np.float32)
        if X.ndim != 2 or X_test.ndim != 2 or X.shape[0] != y.size or \
                X.shape[1] != X_test.shape[1]:
            raise BartError(BART_EINVAL, "X must have one row per class in y, X_test X's columns")
        if n_burn < 0 or n_keep < 1:
            raise BartError(BART_EINVAL, "n_burn must be >= 0 and n_keep >= 1")
        self.n_class = max(int(y.max()) + 1, 2)
        rng = np.random.default_rng([self.seed, 8])
        order = rng.permutation(y.size)
        n_held = min(max(1, int(round(self.holdout * y.size))), y.size - 1)
        held, kept = order[:n_held], order[n_held:]
        Xt = np.ascontiguousarray(X.T)
        Xs = np.ascontiguousarray(X_test.T)
        self.cuts, self.n_cuts = bart_cutpoints(Xt[:, kept], self.K, self.grid)
        Xb = bart_bin(Xt[:, kept], self.cuts, self.n_cuts)
        points = bart_bin(np.concatenate([Xt[:, held], Xs], axis=1), self.cuts, self.n_cuts)
        nt, scores = points.shape[1], None
        for j in range(self.n_class):
            is_j = (y[kept] == j).astype(np.float32)
            # a class that is always or never there still has a finite offset
            offset = NormalDist().inv_cdf((is_j.sum() + 0.5) / (is_j.size + 1.0))
            g = Bart(Xb, is_j, self.n_cuts, ntree=self.ntree, max_depth=self.max_depth,
                     sigma_mu=3.0 / (2.0 * math.sqrt(self.ntree)), nchain=self.nchain,
                     probit=True, probit_offset=offset)
            Xd, _ = g.upload_x(points)
            s = torch.zeros((self.nchain, nt), dtype=torch.float64, device=g.device)
            s2 = torch.zeros_like(s)
            g.step(n_burn, self.seed + j)
            for _ in range(n_keep):
                g.step(1, self.seed + j)
                g.predict_accumulate(Xd, nt, offset, s, s2)
            if g.status():
                raise BartError(BART_EDEVICE, "device error during sampling")
            if scores is None:
                scores = torch.empty((self.nchain, nt, self.n_class), device=g.device)
            scores[:, :, j] = s / n_keep
            g.close()
        self.scores = scores[:, n_held:].contiguous()
        self.held_scores = scores[:, :n_held].contiguous()
        self.held_labels = torch.from_numpy(y[held].astype(np.int64)).to(scores.device)
        self.calibration = Calibration(self.n_class, self.nchain)
        self.losses = self.calibration.fit(self.held_scores, self.held_labels,
                                           self.calibration_steps)
        return self

    def answer(self, y_test=None, k: int = 1) -> ops.LogProb:
        """The calibrated answers at the test points (ops.LogProb); y_test: their
        classes, negative where there is none (one that was not fitted has logp NaN)."""
        import torch

        label = None
        if y_test is not None:
            y = np.asarray(y_test)
            if y.shape != (self.scores.shape[1],) or not np.issubdtype(y.dtype, np.integer):
                raise BartError(BART_EINVAL, "y_test must be a class for each test point")
            label = torch.from_numpy(y.astype(np.int64)).to(self.scores.device)
        return self.calibration.answer(self.scores, label, k=min(k, self.n_class))
