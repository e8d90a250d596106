"""Tuning a model's heads in FP32 or BF16 on the features of an encoder that
stays as it is.

HeadTuner puts the head-tuning operators together as a program uses them: the
encoder's features s (Runtime.features) go through an adapter, a residual
block of layer norm and two dense layers that starts as the identity,

    a = s + W2 silu(W1 norm(s) + b1) + b2,

then through the model's shared layers and, grouped by dataset, its branches
to atom energies; a step takes the mean absolute error of the structures'
energies (the loss of the paper's training), runs the reverse pass and one
AdamW step over all tensors.

The structures of a batch come sorted by dataset (dataset_order), so that the
atoms of a head are consecutive rows.
"""
from __future__ import annotations

import math

import numpy as np


def dataset_order(dataset_id) -> np.ndarray:
    """The order that sorts a batch's structures by dataset, stable."""
    return np.argsort(np.asarray(dataset_id), kind="stable")


SUM_WIDTH = 64


def _sum_levels(ptr):
    """The structures' sums as levels of fixed rows: of each level, which values
    of the level before a row adds, at most SUM_WIDTH consecutive ones of one
    structure; places past them hold the index behind the last value.  The last
    level has one row per structure."""
    begin, count, levels = ptr[:-1], np.diff(ptr), []
    while True:
        total = int(begin[-1] + count[-1]) if len(count) else 0
        last = count.max(initial=0) <= SUM_WIDTH
        rows = np.ones_like(count) if last else -(-count // SUM_WIDTH)
        start = np.cumsum(rows) - rows
        inner = np.arange(rows.sum()) - np.repeat(start, rows)       # the row's place in its structure
        width = max(1, int(count.max(initial=0))) if last else SUM_WIDTH
        first = inner * SUM_WIDTH
        place = first[:, None] + np.arange(width)
        levels.append(np.where(place < np.repeat(count, rows)[:, None], np.repeat(begin, rows)[:, None] + place, total))
        if last:
            return levels
        begin, count = start, rows


class HeadTuner:
    """weights: the model's arrays by name (shared{m}.w, shared{m}.b,
    head{h}.{m}.w, head{h}.{m}.b, as the weight file orders them).  F: the
    width of the features.  dtype: "fp32" or "bf16", of the activations, the
    products' weights and the gradients; masters, sums and atom energies are
    FP32, energies FP64.  adapter: the adapter's inner width (0: none).
    state_bits: 32 or 8, of the optimizer's states."""

    def __init__(self, rt, weights, F, n_heads, n_shared, n_branch, dtype="bf16", adapter=0, lr=6.34e-4,
                 betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, state_bits=32, seed=0):
        import torch
        if dtype not in ("fp32", "bf16"):
            raise ValueError(f"dtype is fp32 or bf16, not {dtype!r}")
        self.rt, self.F, self.n_heads = rt, F, n_heads
        self.n_shared, self.n_branch, self.adapter = n_shared, n_branch, adapter
        self.dtype = torch.float32 if dtype == "fp32" else torch.bfloat16
        dev = rt.device
        init = {}
        if adapter:
            rng = np.random.default_rng(seed)
            init["norm.w"], init["norm.b"] = np.ones(F), np.zeros(F)
            init["adapter0.w"] = rng.standard_normal((adapter, F)) / math.sqrt(F)
            init["adapter0.b"] = np.zeros(adapter)
            init["adapter1.w"], init["adapter1.b"] = np.zeros((F, adapter)), np.zeros(F)
        for m in range(n_shared):
            init[f"shared{m}.w"], init[f"shared{m}.b"] = weights[f"shared{m}.w"], weights[f"shared{m}.b"]
        for m in range(n_branch):       # one stack per branch layer: [heads, out, in]
            for k in "wb":
                init[f"branch{m}.{k}"] = np.stack([weights[f"head{h}.{m}.{k}"] for h in range(n_heads)])
        self.master = {k: torch.as_tensor(np.ascontiguousarray(v), dtype=torch.float32).to(dev)
                       for k, v in init.items()}
        # the weights that the products read: in FP32 the masters themselves
        low = self.dtype == torch.bfloat16
        self.weight = {k: v.to(torch.bfloat16) for k, v in self.master.items()} if low else self.master
        self.grad = {k: torch.zeros_like(v, dtype=self.dtype) for k, v in self.master.items()}
        names = list(self.master)
        self.optimizer = rt.adamw([self.master[k] for k in names], [self.grad[k] for k in names], lr=lr, betas=betas,
                                  eps=eps, weight_decay=weight_decay, state_bits=state_bits,
                                  copies=[self.weight[k] for k in names] if low else None)

    # ---- batches ---------------------------------------------------------
    def batch(self, features, struct_ptr, dataset_id):
        """What a pass needs of a batch: its features [N, F] in the tuner's
        type, its rows by head and by structure."""
        import torch
        ptr, ids = np.asarray(struct_ptr, dtype=np.int64), np.asarray(dataset_id, dtype=np.int64)
        if features.shape != (int(ptr[-1]), self.F):
            raise ValueError(f"features must be [{int(ptr[-1])}, {self.F}], not {list(features.shape)}")
        if len(ids) and (np.any(np.diff(ids) < 0) or ids[0] < 0 or ids[-1] >= self.n_heads):
            raise ValueError("structures must be sorted by dataset id, ids within the heads (dataset_order)")
        cuts = ptr[np.searchsorted(ids, np.arange(self.n_heads + 1))]
        dev = self.rt.device
        return dict(s=features.to(self.dtype).contiguous(), offsets=torch.as_tensor(cuts, dtype=torch.int32).to(dev),
                    ptr=torch.as_tensor(ptr).to(dev), sums=[torch.as_tensor(k).to(dev) for k in _sum_levels(ptr)],
                    structure=torch.as_tensor(np.repeat(np.arange(len(ids)), np.diff(ptr))).to(dev))

    # ---- forward ---------------------------------------------------------
    def _forward(self, b, keep):
        """Atom energies [N, 1] in FP32 and what the reverse pass needs of every
        layer."""
        import torch
        rt, w, kept = self.rt, self.weight, {}
        a = b["s"]
        if self.adapter:
            h, mean, rstd = rt.layer_norm(a, w["norm.w"], w["norm.b"])
            t, z = rt.linear(h, w["adapter0.w"], w["adapter0.b"], activation="silu", keep_preact=True)
            kept.update(h=h, mean=mean, rstd=rstd, t=t, tz=z)
            a = rt.linear(t, w["adapter1.w"], w["adapter1.b"], residual=a)
        layers = []
        x, xz = a, None
        for m in range(self.n_shared):
            y, z = rt.linear(x, w[f"shared{m}.w"], w[f"shared{m}.b"], activation="silu", keep_preact=True)
            layers.append((f"shared{m}", x, xz))
            x, xz = y, z
        for m in range(self.n_branch):
            last = m + 1 == self.n_branch
            y = rt.grouped_linear(x, w[f"branch{m}.w"], b["offsets"], w[f"branch{m}.b"],
                                  activation="none" if last else "silu", keep_preact=not last,
                                  out=torch.empty((len(x), 1), dtype=torch.float32, device=x.device)
                                  if last else None)
            layers.append((f"branch{m}", x, xz))
            x, xz = (y, None) if last else y
        kept["layers"] = layers if keep else None
        return x, kept

    @staticmethod
    def _sum(b, e):
        """Energies of the structures in FP64, each from its own atoms alone,
        the same order in every call."""
        import torch
        v = e.double().view(-1)
        for rows in b["sums"]:
            v = torch.cat([v, v.new_zeros(1)])[rows].sum(1)
        return v

    def energies(self, b):
        return self._sum(b, self._forward(b, False)[0])

    # ---- a step ----------------------------------------------------------
    def gradients(self, b, energy_ref):
        """The loss, mean |E - energy_ref| (energy_ref [structures], or one
        number); its gradients go to self.grad.  Gradients of the features are
        not formed."""
        import torch
        rt, w, g = self.rt, self.weight, self.grad
        want = (len(b["ptr"]) - 1,)
        if tuple(getattr(energy_ref, "shape", ())) not in ((), want):
            raise ValueError(f"energy_ref must be {list(want)}, not {list(energy_ref.shape)}")
        e, kept = self._forward(b, True)
        diff = self._sum(b, e) - energy_ref
        sign = torch.sign(diff) / max(1, diff.numel())
        d = sign[b["structure"]].to(self.dtype).view(-1, 1)
        layers = kept["layers"]
        for k, (name, x, xz) in enumerate(reversed(layers)):
            first = k + 1 == len(layers)
            how = dict(x_activation="none" if xz is None else "silu", x_preact=xz,
                       need_dx=not first or bool(self.adapter), dweight=g[name + ".w"], dbias=g[name + ".b"])
            if name.startswith("branch"):
                d, _, _ = rt.grouped_linear_backward(d, x, w[name + ".w"], b["offsets"], **how)
            else:
                d, _, _ = rt.linear_backward(d, x, w[name + ".w"], **how)
        if self.adapter:
            d, _, _ = rt.linear_backward(d, kept["t"], w["adapter1.w"], x_activation="silu", x_preact=kept["tz"],
                                         dweight=g["adapter1.w"], dbias=g["adapter1.b"])
            d, _, _ = rt.linear_backward(d, kept["h"], w["adapter0.w"], dweight=g["adapter0.w"],
                                         dbias=g["adapter0.b"])
            rt.layer_norm_backward(d, b["s"], w["norm.w"], kept["mean"], kept["rstd"], need_dx=False,
                                   dweight=g["norm.w"], dbias=g["norm.b"])
        return diff.abs().mean()

    def step(self, b, energy_ref, lr=None):
        """One step on a batch; returns the loss before it."""
        loss = self.gradients(b, energy_ref)
        self.optimizer.step(lr)
        return loss

    def weights(self):
        """The tuned heads by the weight file's names (numpy, FP64), without the
        adapter."""
        out = {}
        for k, v in self.master.items():
            a = v.double().cpu().numpy()
            if k.startswith("shared"):
                out[k] = a
            elif k.startswith("branch"):
                m, kind = k[len("branch"):].split(".")
                out.update({f"head{h}.{m}.{kind}": a[h] for h in range(self.n_heads)})
        return out

    def free(self):
        self.optimizer.free()
