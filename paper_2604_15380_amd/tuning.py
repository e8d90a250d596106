"""Tuning a model's heads, or its branch-weighting MLP, in FP32 or BF16 on the
features of an encoder that stays as it is.

HeadTuner puts the head-tuning operators together as a program uses them: the
encoder's features s (Runtime.features) go through an adapter, a residual
block of layer norm and two dense layers that starts as the identity,

    a = s + W2 silu(W1 norm(s) + b1) + b2,

or with group norm over each structure's atoms

    a = s + W2 silu(norm(W1 s + b1)) + b2,

then through the model's shared layers and, grouped by dataset, its branches
to atom energies; a step takes the mean absolute error of the structures'
energies (the loss of the paper's training), runs the reverse pass and one
AdamW step over all tensors.

GateTuner does the same for the gate over the heads: compositions -> dense SiLU
layers -> softmax weights of the k largest heads -> blended energies; a step
takes the mean squared error of the energies (the loss of the paper's branch
weighting) and the gate's balance loss.

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


def _optimized(tuner, init, max_norm, **how):
    """A tuner's masters, the weights that the products read (in FP32 the masters
    themselves), their gradients, and the optimizer over all of them."""
    import torch
    dev = tuner.rt.device
    tuner.master = {k: torch.as_tensor(np.ascontiguousarray(v), dtype=torch.float32).to(dev) for k, v in init.items()}
    low = tuner.dtype == torch.bfloat16
    tuner.weight = {k: v.to(torch.bfloat16) for k, v in tuner.master.items()} if low else tuner.master
    tuner.grad = {k: torch.zeros_like(v, dtype=tuner.dtype) for k, v in tuner.master.items()}
    names = list(tuner.master)
    grads = [tuner.grad[k] for k in names]
    tuner.optimizer = tuner.rt.adamw([tuner.master[k] for k in names], grads,
                                     copies=[tuner.weight[k] for k in names] if low else None, **how)
    tuner.max_norm = max_norm
    tuner.grad_norm = tuner.rt.grad_norm(grads) if max_norm is not None else None


def _optimize(tuner, lr):
    """The optimizer's step on the gradients, clipped where the tuner clips."""
    factor = None
    if tuner.grad_norm is not None:
        tuner.norm, factor = tuner.grad_norm.compute(tuner.max_norm)
    tuner.optimizer.step(lr, grad_scale=factor)


def _free(tuner):
    tuner.optimizer.free()
    if tuner.grad_norm is not None:
        tuner.grad_norm.free()


class HeadTuner:
    """weights: the model's arrays by name (shared{m}.w, shared{m}.b,
    head{h}.{m}.w, head{h}.{m}.b, as the weight file orders them).  F: the
    width of the features.  dtype: "fp32" or "bf16", of the activations, the
    products' weights and the gradients; masters, sums and atom energies are
    FP32, energies FP64.  adapter: the adapter's inner width (0: none);
    adapter_norm: "layer", of each atom's features, or "group", of adapter_groups
    groups of the inner columns over a structure's atoms.  state_bits: 32 or 8,
    of the optimizer's states.  max_norm: gradients are clipped to this global
    norm (None: not)."""

    def __init__(self, rt, weights, F, n_heads, n_shared, n_branch, dtype="bf16", adapter=0, lr=6.34e-4,
                 betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, state_bits=32, seed=0, adapter_norm="layer",
                 adapter_groups=8, max_norm=None):
        import torch
        if dtype not in ("fp32", "bf16"):
            raise ValueError(f"dtype is fp32 or bf16, not {dtype!r}")
        if adapter_norm not in ("layer", "group"):
            raise ValueError(f"adapter_norm is layer or group, not {adapter_norm!r}")
        self.rt, self.F, self.n_heads = rt, F, n_heads
        self.n_shared, self.n_branch, self.adapter = n_shared, n_branch, adapter
        self.groups = 0         # of the adapter's group norm (0: it has none)
        if adapter and adapter_norm == "group":
            if adapter_groups < 1 or adapter % adapter_groups:
                raise ValueError(f"{adapter_groups} groups do not divide {adapter} columns")
            self.groups = adapter_groups
        self.dtype = torch.float32 if dtype == "fp32" else torch.bfloat16
        init = {}
        if adapter:
            rng = np.random.default_rng(seed)
            width = adapter if self.groups else F
            init["norm.w"], init["norm.b"] = np.ones(width), np.zeros(width)
            init["adapter0.w"] = rng.standard_normal((adapter, F)) / math.sqrt(F)
            init["adapter0.b"] = np.zeros(adapter)
            init["adapter1.w"], init["adapter1.b"] = np.zeros((F, adapter)), np.zeros(F)
        for m in range(n_shared):
            init[f"shared{m}.w"], init[f"shared{m}.b"] = weights[f"shared{m}.w"], weights[f"shared{m}.b"]
        for m in range(n_branch):       # one stack per branch layer: [heads, out, in]
            for k in "wb":
                init[f"branch{m}.{k}"] = np.stack([weights[f"head{h}.{m}.{k}"] for h in range(n_heads)])
        _optimized(self, init, max_norm, lr=lr, betas=betas, eps=eps, weight_decay=weight_decay, state_bits=state_bits)

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
                    ptr=torch.as_tensor(ptr).to(dev), samples=torch.as_tensor(ptr, dtype=torch.int32).to(dev),
                    longest=int(np.diff(ptr).max(initial=0)), sums=[torch.as_tensor(k).to(dev) for k in _sum_levels(ptr)],
                    structure=torch.as_tensor(np.repeat(np.arange(len(ids)), np.diff(ptr))).to(dev))

    # ---- forward ---------------------------------------------------------
    def _forward(self, b, keep):
        """Atom energies [N, 1] in FP32 and what the reverse pass needs of every
        layer."""
        import torch
        rt, w, kept = self.rt, self.weight, {}
        a = b["s"]
        if self.groups:
            t = rt.linear(a, w["adapter0.w"], w["adapter0.b"])
            h, mean, rstd = rt.group_norm(t, w["norm.w"], w["norm.b"], self.groups, offsets=b["samples"],
                                          activation="silu", max_rows=b["longest"])
            kept.update(t=t, h=h, mean=mean, rstd=rstd)
            a = rt.linear(h, w["adapter1.w"], w["adapter1.b"], residual=a)
        elif self.adapter:
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
        if self.groups:
            d, _, _ = rt.linear_backward(d, kept["h"], w["adapter1.w"], dweight=g["adapter1.w"], dbias=g["adapter1.b"])
            d, _, _ = rt.group_norm_backward(d, kept["t"], w["norm.w"], w["norm.b"], kept["mean"], kept["rstd"],
                                             self.groups, offsets=b["samples"], activation="silu", max_rows=b["longest"],
                                             dx=d, dweight=g["norm.w"], dbias=g["norm.b"])
            rt.linear_backward(d, b["s"], w["adapter0.w"], need_dx=False, dweight=g["adapter0.w"], dbias=g["adapter0.b"])
        elif self.adapter:
            d, _, _ = rt.linear_backward(d, kept["t"], w["adapter1.w"], x_activation="silu", x_preact=kept["tz"],
                                         dweight=g["adapter1.w"], dbias=g["adapter1.b"])
            d, _, _ = rt.linear_backward(d, kept["h"], w["adapter0.w"], dweight=g["adapter0.w"],
                                         dbias=g["adapter0.b"])
            rt.layer_norm_backward(d, b["s"], w["norm.w"], kept["mean"], kept["rstd"], need_dx=False,
                                   dweight=g["norm.w"], dbias=g["norm.b"])
        return diff.abs().mean()

    def step(self, b, energy_ref, lr=None):
        """One step on a batch; returns the loss before it.  With max_norm the
        gradients' norm before clipping is in self.norm."""
        loss = self.gradients(b, energy_ref)
        _optimize(self, lr)
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
        _free(self)


def head_energies(rt, model, graph, precision="fp32"):
    """Every head's energy of every structure, [structures, heads] in FP64: what
    GateTuner blends."""
    import torch
    ids = torch.empty(graph.n_struct, dtype=torch.int32, device=rt.device)
    out = torch.empty((graph.n_struct, model.info["n_heads"]), dtype=torch.float64, device=rt.device)
    for h in range(model.info["n_heads"]):
        out[:, h] = rt.forward(model, graph, precision, ids.fill_(h))
    return out


class GateTuner:
    """Tunes the branch-weighting MLP, which weights the heads of a structure by
    its composition.  weights: the model's arrays blend{m}.w, blend{m}.b of its
    n_layers layers.  k: heads that are kept of a structure (None: all), with
    their weights as they are or, with normalize, adding up to 1.  balance: the
    coefficient of the gate's balance loss.  dtype: "fp32" or "bf16", of the
    activations, the products' weights and the gradients.  max_norm: gradients
    are clipped to this global norm (None: not).  It starts as the model's own
    blend (painn_forward_blend with no threshold, for k = None)."""

    def __init__(self, rt, weights, n_layers, k=None, normalize=False, balance=0.0, dtype="fp32", lr=6.34e-4,
                 betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, state_bits=32, max_norm=None):
        import torch
        if dtype not in ("fp32", "bf16"):
            raise ValueError(f"dtype is fp32 or bf16, not {dtype!r}")
        self.n_species, self.n_heads = weights["blend0.w"].shape[1], weights[f"blend{n_layers - 1}.w"].shape[0]
        self.k = self.n_heads if k is None else k
        if not 0 < self.k <= self.n_heads:
            raise ValueError(f"k must be within 1 and {self.n_heads} heads, not {k}")
        self.rt, self.n_layers, self.normalize, self.balance = rt, n_layers, normalize, balance
        self.whole = bool(normalize) or self.k == self.n_heads      # a structure's weights add up to 1
        self.dtype = torch.float32 if dtype == "fp32" else torch.bfloat16
        init = {f"blend{m}.{c}": weights[f"blend{m}.{c}"] for m in range(n_layers) for c in "wb"}
        _optimized(self, init, max_norm, lr=lr, betas=betas, eps=eps, weight_decay=weight_decay, state_bits=state_bits)

    def batch(self, species, struct_ptr, head_energies):
        """What a pass needs of a batch: its compositions (the fraction of a
        structure's atoms of each species) and its heads' energies [structures,
        heads] (head_energies)."""
        import torch
        ptr, z = np.asarray(struct_ptr, dtype=np.int64), np.asarray(species, dtype=np.int64)
        n = len(ptr) - 1
        if tuple(head_energies.shape) != (n, self.n_heads):
            raise ValueError(f"head_energies must be [{n}, {self.n_heads}], not {list(head_energies.shape)}")
        if len(z) and (z.min() < 0 or z.max() >= self.n_species):
            raise ValueError(f"species must be within [0, {self.n_species})")
        count = np.zeros((n, self.n_species))
        np.add.at(count, (np.repeat(np.arange(n), np.diff(ptr)), z), 1.0)
        count /= np.maximum(1, np.diff(ptr))[:, None]
        return dict(x=torch.as_tensor(count).to(self.rt.device).to(self.dtype), heads=head_energies.double())

    def _forward(self, b):
        """The gate, and every layer's input, its pre-activations and the logits."""
        x, xz, layers = b["x"], None, []
        for m in range(self.n_layers):
            last = m + 1 == self.n_layers
            y = self.rt.linear(x, self.weight[f"blend{m}.w"], self.weight[f"blend{m}.b"],
                               activation="none" if last else "silu", keep_preact=not last)
            layers.append((f"blend{m}", x, xz))
            x, xz = (y, None) if last else y
        return self.rt.gate(x, self.k, normalize=self.normalize), x, layers

    def _blend(self, b, gate):
        """Energies, and what the energies of the heads that were chosen give to
        the gate's gradient (0 for none).  Where a structure's weights add up to
        1, a value that is taken off all its heads changes neither: the FP32
        weights then meet the differences of the heads alone, in which total
        energies, 1e5 times as large, leave no rounding."""
        import torch
        none = gate.indices < 0
        e = b["heads"].gather(1, gate.indices.clamp_min(0).long())
        about = e[:, :1] if self.whole else torch.zeros_like(e[:, :1])
        e = torch.where(none, torch.zeros_like(e), e - about)
        energies = (gate.weights.double() * e).sum(1)
        part = e - energies[:, None] if self.whole else e
        # (a structure without a head has no energy)
        about = torch.where(none[:, 0], torch.zeros_like(energies), about[:, 0])
        return about + energies, torch.where(none, torch.zeros_like(e), part)

    def energies(self, b):
        return self._blend(b, self._forward(b)[0])[0]

    def gradients(self, b, energy_ref):
        """The loss, mean (E - energy_ref)^2 + balance times the gate's balance
        loss; its gradients go to self.grad, the gate to self.gate."""
        import torch
        want = (len(b["x"]),)
        if tuple(getattr(energy_ref, "shape", ())) not in ((), want):
            raise ValueError(f"energy_ref must be {list(want)}, not {list(energy_ref.shape)}")
        gate, logits, layers = self._forward(b)
        self.gate = gate
        energies, heads = self._blend(b, gate)
        diff = energies - energy_ref
        n = max(1, diff.numel())
        dw = (diff[:, None] * heads * (2.0 / n)).float()
        # (in a BF16 batch dlogits is rounded as every gradient)
        d = self.rt.gate_backward(dw, logits, gate, balance=self.balance)
        for k, (name, x, xz) in enumerate(reversed(layers)):
            d, _, _ = self.rt.linear_backward(d, x, self.weight[name + ".w"], x_activation="none" if xz is None else "silu",
                                              x_preact=xz, need_dx=k + 1 < len(layers), dweight=self.grad[name + ".w"],
                                              dbias=self.grad[name + ".b"])
        return (diff * diff).sum() / n + self.balance * gate.loss.double()

    def step(self, b, energy_ref, lr=None):
        """One step on a batch; returns the loss before it.  With max_norm the
        gradients' norm before clipping is in self.norm."""
        loss = self.gradients(b, energy_ref)
        _optimize(self, lr)
        return loss

    def weights(self):
        """The tuned MLP by the weight file's names (numpy, FP64)."""
        return {k: v.double().cpu().numpy() for k, v in self.master.items()}

    def free(self):
        _free(self)
