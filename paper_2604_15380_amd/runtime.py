"""Torch-facing convenience layer over the C ABI: device memory and the HIP
stream come from torch; every computation runs in libpainn.so."""
from __future__ import annotations

import ctypes
import sys

import numpy as np

from . import binding as B


def _hip():
    return ctypes.CDLL("libamdhip64.so")


def copy_from_device(dst, src_ptr: int, nbytes: int) -> None:
    """Copy `nbytes` from a library-owned device pointer into a torch tensor."""
    import torch
    if nbytes == 0:
        return
    torch.cuda.synchronize(dst.device)
    h = _hip()
    h.hipMemcpy.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int]
    err = h.hipMemcpy(dst.data_ptr(), src_ptr, nbytes, 3)   # hipMemcpyDeviceToDevice
    if err != 0:
        raise RuntimeError(f"hipMemcpy failed ({err})")


class Model:
    def __init__(self, rt: "Runtime", handle: int):
        self.rt, self.handle = rt, handle
        self.info = B.painn_model_info(handle)
        opts = B.painn_model_options(handle)
        self.has_blend = opts["has_blend"]
        self.max_neighbors = opts["max_neighbors"]

    def free(self):
        if self.handle:
            B.painn_model_free(self.handle)
            self.handle = 0


class Graph:
    def __init__(self, rt: "Runtime", handle: int, inputs):
        self.rt, self.handle, self.inputs = rt, handle, inputs
        self.refresh()

    def refresh(self):
        c = B.painn_graph_csr(self.handle)
        self.n_edges, self.n_atoms, self.n_struct = c["n_edges"], c["n_atoms"], c["n_struct"]
        self._ptrs = c

    def csr(self):
        """(row_ptr [N+1], col [E], shift [E,3]) as CPU numpy int64 arrays."""
        import torch
        dev = self.rt.device
        rp = torch.empty(self.n_atoms + 1, dtype=torch.int32, device=dev)
        col = torch.empty(self.n_edges, dtype=torch.int32, device=dev)
        sh = torch.empty(self.n_edges, dtype=torch.int32, device=dev)
        copy_from_device(rp, self._ptrs["row_ptr"], 4 * (self.n_atoms + 1))
        copy_from_device(col, self._ptrs["col"], 4 * self.n_edges)
        copy_from_device(sh, self._ptrs["shift"], 4 * self.n_edges)
        sh_np = sh.cpu().numpy().view(np.int8).reshape(-1, 4)[:, :3].astype(np.int64)
        return rp.cpu().numpy().astype(np.int64), col.cpu().numpy().astype(np.int64), sh_np

    def free(self):
        if self.handle:
            B.painn_graph_free(self.handle)
            self.handle = 0


class AdamW:
    """AdamW over many tensors, one launch per step (painn_adamw_*).

    The optimizer reads `grads` and writes `params` (and `copies`) in place.
    state_bits 8 holds the moments as e4m3 codes of m and sqrt(v) with one
    FP32 scale per 256 values: m[k] and v[k] are then torch.float8_e4m3fn, and
    the values are m[k].float() * m_scale[k] (each scale repeated 256 times)
    and the square of v[k].float() * v_scale[k].  Codes are rounded to nearest,
    so that over many steps most second moments move with their block only
    (painn.h has the figures)."""

    def __init__(self, rt, params, grads, lr=6.34e-4, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01,
                 state_bits=32, copies=None, state=None, steps=0):
        import torch
        if state_bits not in (8, 32):
            raise ValueError("state_bits is 8 or 32")
        params, grads = list(params), list(grads)
        copies = list(copies) if copies is not None else [None] * len(params)
        if not len(params) == len(grads) == len(copies):
            raise ValueError("params, grads and copies differ in length")
        gt = grads[0].dtype if grads else torch.float32
        if gt not in _precisions():
            raise ValueError(f"gradients are float32 or bfloat16, not {gt}")
        small = state_bits == 8
        held = torch.float8_e4m3fn if small else torch.float32
        blocks = [-(-p.numel() // 256) for p in params]
        if state is None:
            def zeros(sizes, dtype):
                return [torch.zeros(n * (1 if dtype is held and small else 4), dtype=torch.uint8,
                                    device=rt.device).view(dtype) for n in sizes]
            values = [p.numel() for p in params]
            state = dict(m=zeros(values, held), v=zeros(values, held))
            if small:
                state.update(m_scale=zeros(blocks, torch.float32), v_scale=zeros(blocks, torch.float32))
        self.rt, self.params, self.grads, self.copies = rt, params, grads, copies
        self.state_bits, self.lr = state_bits, lr
        self.m, self.v = list(state["m"]), list(state["v"])
        self.m_scale = list(state["m_scale"]) if small else None
        self.v_scale = list(state["v_scale"]) if small else None
        # a field per list, as painn_adamw_tensor orders them
        lists = [("param", params, torch.float32, 1), ("grad", grads, gt, 1), ("copy", copies, torch.bfloat16, 1),
                 ("m", self.m, held, 1), ("v", self.v, held, 1)]
        if small:
            lists += [("m_scale", self.m_scale, torch.float32, 256), ("v_scale", self.v_scale, torch.float32, 256)]
        sizes = [p.numel() for p in params]
        fields, dev = [sizes], rt.device
        for name, arrays, dtype, per in lists:
            if len(arrays) != len(sizes):
                raise ValueError(f"{len(arrays)} arrays of {name} for {len(sizes)} tensors")
            ptrs = []
            for k, (a, n) in enumerate(zip(arrays, sizes)):
                if a is None and name == "copy":
                    ptrs.append(0)
                    continue
                n = -(-n // per)
                if a.dtype is not dtype or a.numel() != n or not a.is_contiguous() or a.device != dev:
                    raise ValueError(f"tensor {k}: {name} must be contiguous {dtype} of {n} values on {dev}")
                ptrs.append(a.data_ptr())
            fields.append(ptrs)
        while len(fields) < 8:
            fields.append([0] * len(sizes))
        self.handle = 0
        cfg = dict(beta1=betas[0], beta2=betas[1], eps=eps, weight_decay=weight_decay, state_bits=state_bits,
                   grad_precision=B.PAINN_BF16 if gt == torch.bfloat16 else B.PAINN_FP32, steps=steps)
        cur = rt._enter()
        self.handle = B.painn_adamw_create(rt.ctx, B.adamw_tensors(fields), cfg)
        rt._leave(cur, ())

    def step(self, lr=None):
        """One step on the gradients as they are now, at `lr` or the one given
        at the start."""
        cur = self.rt._enter()
        B.painn_adamw_step(self.rt.ctx, self.handle, self.lr if lr is None else lr)
        if cur is not None:
            self.rt._leave(cur, [t for a in (self.params, self.grads, self.copies, self.m, self.v,
                                             self.m_scale or (), self.v_scale or ()) for t in a if t is not None])

    @property
    def steps(self):
        return B.painn_adamw_steps(self.handle)

    def state(self):
        """The states as they are held, for a later AdamW(..., state=, steps=)."""
        d = dict(m=self.m, v=self.v)
        if self.state_bits == 8:
            d.update(m_scale=self.m_scale, v_scale=self.v_scale)
        return d

    def free(self):
        if self.handle:
            B.painn_adamw_free(self.handle)
        self.handle = 0

    def __del__(self):
        if getattr(self, "handle", 0) and sys is not None and not sys.is_finalizing():
            self.free()


_NAMES = {}


def _precisions():
    """torch type -> precision, of the operators for tuning heads."""
    if not _NAMES:
        import torch
        _NAMES.update({torch.float32: B.PAINN_FP32, torch.bfloat16: B.PAINN_BF16})
    return _NAMES


class Runtime:
    """One library context on a torch CUDA (HIP) device and its current stream."""

    def __init__(self, device: int = 0):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU: the HIP library has no CPU path")
        self.device = torch.device("cuda", device)
        self.stream = torch.cuda.current_stream(self.device)
        self.ctx = B.painn_create(device, self.stream.cuda_stream)
        self._stream_id = self.stream.cuda_stream

    # ---- inputs ----------------------------------------------------------
    def upload_batch(self, batch):
        """Copy a synth.Batch (numpy) to device tensors."""
        import torch
        d = self.device
        return dict(
            n_struct=batch.n_struct, n_atoms=batch.n_atoms,
            struct_ptr=torch.from_numpy(np.ascontiguousarray(batch.struct_ptr, dtype=np.int32)).to(d),
            pos=torch.from_numpy(np.ascontiguousarray(batch.pos, dtype=np.float64)).to(d),
            species=torch.from_numpy(np.ascontiguousarray(batch.species, dtype=np.int32)).to(d),
            cell=torch.from_numpy(np.ascontiguousarray(batch.cell, dtype=np.float64)).to(d),
            pbc=torch.from_numpy(np.ascontiguousarray(batch.pbc, dtype=np.uint8)).to(d),
            dataset_id=torch.from_numpy(np.ascontiguousarray(batch.dataset_id, dtype=np.int32)).to(d),
            any_pbc=bool(np.any(batch.pbc)),
        )

    # ---- model / graph / forward ----------------------------------------
    def load_model(self, src) -> Model:
        if isinstance(src, (bytes, bytearray)):
            return Model(self, B.painn_model_load_buffer(self.ctx, bytes(src)))
        return Model(self, B.painn_model_load(self.ctx, str(src)))

    def build_graph(self, inp: dict, cutoff: float, graph: Graph | None = None,
                    max_neighbors: int = 0) -> Graph:
        """Radius graph of an uploaded batch; max_neighbors > 0 keeps that
        many nearest neighbours per receiver (a capped model needs its cap)."""
        ptr = lambda t: t.data_ptr() if t is not None and t.numel() else None
        use_pbc = inp.get("any_pbc", True)
        h = B.painn_build_graph_capped(self.ctx, inp["n_struct"], inp["n_atoms"], ptr(inp["struct_ptr"]),
                                       ptr(inp["pos"]), ptr(inp["species"]),
                                       ptr(inp["cell"]) if use_pbc else None,
                                       ptr(inp["pbc"]) if use_pbc else None, cutoff, max_neighbors,
                                       graph.handle if graph else None)
        if graph is not None:
            graph.inputs = inp
            graph.refresh()
            return graph
        return Graph(self, h, inp)

    def forward(self, model: Model, graph: Graph, precision="fp32", dataset_id=None, out=None):
        import torch
        prec = B.PRECISIONS[precision] if isinstance(precision, str) else precision
        if out is None:
            out = torch.empty(graph.n_struct, dtype=torch.float64, device=self.device)
        ds = dataset_id.data_ptr() if dataset_id is not None and dataset_id.numel() else None
        B.painn_forward(self.ctx, model.handle, graph.handle, ds, prec,
                        out.data_ptr() if out.numel() else None)
        return out

    def forward_blend(self, model: Model, graph: Graph, precision="fp32", skip=0.0, out=None,
                      weights=None):
        """Energies with every head blended by the model's branch-weighting
        MLP; heads with weight < skip are left out.  `weights` (optional)
        receives the [B, n_heads] head weights."""
        import torch
        prec = B.PRECISIONS[precision] if isinstance(precision, str) else precision
        if out is None:
            out = torch.empty(graph.n_struct, dtype=torch.float64, device=self.device)
        B.painn_forward_blend(self.ctx, model.handle, graph.handle, prec, skip,
                              out.data_ptr() if out.numel() else None,
                              weights.data_ptr() if weights is not None and weights.numel() else None)
        return out

    def forces(self, model: Model, graph: Graph, precision="fp32", dataset_id=None, energies=None,
               forces=None):
        """Energies [B] and forces -dE/dx [N, 3] (float64) by the reverse pass."""
        import torch
        prec = B.PRECISIONS[precision] if isinstance(precision, str) else precision
        if energies is None:
            energies = torch.empty(graph.n_struct, dtype=torch.float64, device=self.device)
        if forces is None:
            forces = torch.empty((graph.n_atoms, 3), dtype=torch.float64, device=self.device)
        ds = dataset_id.data_ptr() if dataset_id is not None and dataset_id.numel() else None
        B.painn_forces(self.ctx, model.handle, graph.handle, ds, prec,
                       energies.data_ptr() if energies.numel() else None,
                       forces.data_ptr() if forces.numel() else None)
        return energies, forces

    def forces_blend(self, model: Model, graph: Graph, precision="fp32", skip=0.0, energies=None,
                     forces=None, weights=None):
        """Energies and forces with every head blended by the model's
        branch-weighting MLP (heads with weight < skip left out)."""
        import torch
        prec = B.PRECISIONS[precision] if isinstance(precision, str) else precision
        if energies is None:
            energies = torch.empty(graph.n_struct, dtype=torch.float64, device=self.device)
        if forces is None:
            forces = torch.empty((graph.n_atoms, 3), dtype=torch.float64, device=self.device)
        B.painn_forces_blend(self.ctx, model.handle, graph.handle, prec, skip,
                             energies.data_ptr() if energies.numel() else None,
                             forces.data_ptr() if forces.numel() else None,
                             weights.data_ptr() if weights is not None and weights.numel() else None)
        return energies, forces

    def features(self, model: Model, graph: Graph, layer: int, precision="fp64"):
        import torch
        prec = B.PRECISIONS[precision] if isinstance(precision, str) else precision
        F = model.info["F"]
        s = torch.empty((graph.n_atoms, F), dtype=torch.float64, device=self.device)
        v = torch.empty((graph.n_atoms, 3, F), dtype=torch.float64, device=self.device)
        B.painn_forward_features(self.ctx, model.handle, graph.handle, prec, layer,
                                 s.data_ptr() if s.numel() else None,
                                 v.data_ptr() if v.numel() else None)
        return s, v

    # ---- operators for tuning heads (FP32, BF16) ---------------------------
    # They run on the context's stream, like every call; where torch's current
    # stream is another one, the two wait for each other, so that the caller
    # sees the order of its own stream.
    def _enter(self):
        import torch
        if torch._C._cuda_getCurrentRawStream(self.device.index) == self._stream_id:
            return None
        cur = torch.cuda.current_stream(self.device)
        self.stream.wait_stream(cur)
        return cur

    def _leave(self, cur, tensors):
        if cur is None:
            return
        for t in tensors:
            if t is not None:
                t.record_stream(self.stream)
        cur.wait_stream(self.stream)

    def _precision(self, x):
        try:
            return _precisions()[x.dtype]
        except KeyError:
            raise ValueError(f"the operators take float32 or bfloat16, not {x.dtype}") from None

    def _rows(self, t, name, dtype, rows, cols):
        """(pointer, row stride) of a matrix whose rows are contiguous; (0, 0)
        for None."""
        if t is None:
            return 0, 0
        if t.dtype is not dtype or t.device != self.device:
            raise ValueError(f"{name} must be {dtype} on {self.device}, not {t.dtype} on {t.device}")
        if t.shape != (rows, cols):
            raise ValueError(f"{name} must be [{rows}, {cols}], not {list(t.shape)}")
        ld, step = t.stride()
        if rows <= 1 and ld < cols:
            ld = cols
        if (step != 1 and cols > 1) or ld < cols:
            raise ValueError(f"{name} must have contiguous rows that do not overlap (strides {t.stride()})")
        return t.data_ptr(), ld

    def _whole(self, t, name, dtype, shape):
        """Pointer of a contiguous tensor; 0 for None."""
        if t is None:
            return 0
        if t.dtype is not dtype or t.device != self.device or t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {list(shape)} on {self.device}, "
                             f"not {t.dtype} {list(t.shape)} on {t.device}")
        return t.data_ptr()

    def layer_norm(self, x, weight, bias, eps=1e-5, out=None):
        """(y, mean, rstd) of every row of x [rows, cols]; mean and rstd [rows]
        are FP32 and go to layer_norm_backward.  `out` may be x."""
        import torch
        prec, t = self._precision(x), x.dtype
        if x.dim() != 2:
            raise ValueError("x must be [rows, cols]")
        n, c = x.shape
        px, ldx = self._rows(x, "x", t, n, c)
        pw, pb = self._whole(weight, "weight", t, (c,)), self._whole(bias, "bias", t, (c,))
        if out is None:
            out = x.new_empty((n, c))
        py, ldy = self._rows(out, "out", t, n, c)
        stats = x.new_empty((2, n), dtype=torch.float32)
        mean, rstd = stats.unbind()
        cur = self._enter()
        B.painn_layer_norm(self.ctx, prec, n, c, px, ldx, pw, pb, eps, py, ldy, mean.data_ptr(), rstd.data_ptr())
        if cur is not None:
            self._leave(cur, (x, weight, bias, out, stats))
        return out, mean, rstd

    def layer_norm_backward(self, dy, x, weight, mean, rstd, dx=None, dweight=None, dbias=None, need_dx=True):
        """(dx, dweight, dbias) from dy and the forward's x, mean and rstd; dx
        is None without need_dx and may be given as dy."""
        import torch
        prec, t = self._precision(x), x.dtype
        if x.dim() != 2:
            raise ValueError("x must be [rows, cols]")
        n, c = x.shape
        px, ldx = self._rows(x, "x", t, n, c)
        pd, ldd = self._rows(dy, "dy", t, n, c)
        pw = self._whole(weight, "weight", t, (c,))
        pm, pr = (self._whole(a, k, torch.float32, (n,)) for a, k in ((mean, "mean"), (rstd, "rstd")))
        if need_dx and dx is None:
            dx = x.new_empty((n, c))
        dweight = torch.empty_like(weight) if dweight is None else dweight
        dbias = torch.empty_like(weight) if dbias is None else dbias
        po, ldo = self._rows(dx, "dx", t, n, c)
        pg, pb = self._whole(dweight, "dweight", t, (c,)), self._whole(dbias, "dbias", t, (c,))
        cur = self._enter()
        B.painn_layer_norm_backward(self.ctx, prec, n, c, pd, ldd, px, ldx, pw, pm, pr, po, ldo, pg, pb)
        if cur is not None:
            self._leave(cur, (dy, x, weight, mean, rstd, dx, dweight, dbias))
        return dx, dweight, dbias

    def _activation(self, name):
        try:
            return B.ACTIVATIONS[name]
        except KeyError:
            raise ValueError(f"unknown activation {name!r}: one of {', '.join(B.ACTIVATIONS)}") from None

    def _shapes(self, x, weight, offsets):
        """(rows, d_in, d_out, leading shape of the weights, groups, offsets' pointer)"""
        import torch
        if x.dim() != 2 or weight.dim() != (2 if offsets is None else 3):
            raise ValueError("x must be [rows, d_in] and weight " + ("[d_out, d_in]" if offsets is None
                                                                     else "[groups, d_out, d_in]"))
        n, i = x.shape
        if offsets is None:
            return n, i, weight.shape[0], (), 0, 0
        g, o, _ = weight.shape
        return n, i, o, (g,), g, self._whole(offsets, "offsets", torch.int32, (g + 1,))

    @staticmethod
    def _kept(x, rows, cols):
        """An array for the reverse pass and its row stride.  Beyond the caches'
        size rows start at whole 128-byte lines: a line in two rows would go to
        memory twice (65,502 x 776 BF16 in 16 groups, SiLU: 178 -> 168 us)."""
        size = x.element_size()
        ld = cols
        if rows * cols * size > 32 << 20 and cols * size % 128:
            ld = -(-cols * size // 128) * 128 // size
        z = x.new_empty((rows, ld))
        return (z if ld == cols else z[:, :cols]), ld

    def _dense(self, x, weight, offsets, bias, activation, residual, keep_preact, out):
        prec, t = self._precision(x), x.dtype
        n, i, o, lead, groups, po = self._shapes(x, weight, offsets)
        act = self._activation(activation)
        px, ldx = self._rows(x, "x", t, n, i)
        pw = self._whole(weight, "weight", t, lead + (o, i))
        pb = self._whole(bias, "bias", t, lead + (o,))
        pr, ldr = self._rows(residual, "residual", t, n, o)
        full = out is not None and _precisions().get(out.dtype) == B.PAINN_FP32
        if out is None:
            out = x.new_empty((n, o))
        py, ldy = self._rows(out, "out", out.dtype if full else t, n, o)
        z, pz, ldz = None, 0, 0
        if keep_preact:
            z, ldz = self._kept(x, n, o)
            pz = z.data_ptr()
        cur = self._enter()
        a = B.linear_args(prec, act, n, i, o, px, ldx, pw, pb, pr, ldr, py, ldy, pz, ldz, full, 0)
        if groups:
            B.painn_grouped_linear(self.ctx, a, groups, po)
        else:
            B.painn_linear(self.ctx, a)
        if cur is not None:
            self._leave(cur, (x, weight, offsets, bias, residual, out, z))
        return (out, z) if keep_preact else out

    def linear(self, x, weight, bias=None, activation="none", residual=None, keep_preact=False, out=None):
        """y = activation(x weight^T + bias) + residual; x [rows, d_in], weight
        [d_out, d_in].  keep_preact: (y, z), z the activation's input, for
        linear_backward (a large z has gaps between its rows).  `residual` may
        be `out`.  A float32 `out` takes a BF16 layer's results unrounded (a
        readout's, of a few columns)."""
        return self._dense(x, weight, None, bias, activation, residual, keep_preact, out)

    def grouped_linear(self, x, weight, offsets, bias=None, activation="none", residual=None, keep_preact=False,
                       out=None):
        """linear with weight [groups, d_out, d_in] and bias [groups, d_out]:
        group g has the rows offsets[g] .. offsets[g+1] (int32 on the GPU).
        Rows of no group are left as they are in `out` (undefined in a new
        one)."""
        if offsets is None:
            raise ValueError("offsets is missing")
        return self._dense(x, weight, offsets, bias, activation, residual, keep_preact, out)

    def _dense_backward(self, dy, x, weight, offsets, activation, preact, x_activation, x_preact, need_dx, dx,
                        dweight, dbias, dz_remainders):
        import torch
        prec, t = self._precision(x), x.dtype
        n, i, o, lead, groups, po = self._shapes(x, weight, offsets)
        act, x_act = self._activation(activation), self._activation(x_activation)
        if act and preact is None:
            raise ValueError(f"preact is missing for activation {activation!r}")
        if x_act and need_dx and x_preact is None:
            raise ValueError(f"x_preact is missing for x_activation {x_activation!r}")
        pdy, lddy = self._rows(dy, "dy", t, n, o)
        pz, ldz = self._rows(preact, "preact", t, n, o)
        px, ldx = self._rows(x, "x", t, n, i)
        pw = self._whole(weight, "weight", t, lead + (o, i))
        pxz, ldxz = self._rows(x_preact, "x_preact", t, n, i)
        if need_dx and dx is None:
            dx = x.new_empty((n, i))
        if dweight is None:
            dweight = torch.empty_like(weight)
        if dbias is None:
            dbias = x.new_empty(lead + (o,))
        pdx, lddx = self._rows(dx, "dx", t, n, i)
        pdw = self._whole(dweight, "dweight", t, lead + (o, i))
        pdb = self._whole(dbias, "dbias", t, lead + (o,))
        cur = self._enter()
        a = B.linear_backward_args(prec, act, n, i, o, pdy, lddy, pz, ldz, px, ldx, pw, pxz, ldxz, x_act, dz_remainders,
                                   pdx, lddx, pdw, pdb)
        if groups:
            B.painn_grouped_linear_backward(self.ctx, a, groups, po)
        else:
            B.painn_linear_backward(self.ctx, a)
        if cur is not None:
            self._leave(cur, (dy, x, weight, offsets, preact, x_preact, dx, dweight, dbias))
        return dx, dweight, dbias

    def linear_backward(self, dy, x, weight, activation="none", preact=None, x_activation="none", x_preact=None,
                        need_dx=True, dx=None, dweight=None, dbias=None, dz_remainders=False):
        """(dx, dweight, dbias) of linear.  preact: the forward's z, needed with
        an activation.  With x_activation and x_preact (x =
        x_activation(x_preact)), dx is the gradient of x_preact.  The
        residual's gradient is dy.  In BF16 with an activation, dy times its
        slope is rounded to BF16 before the products where it has more than
        8,192 values (dbias is not); with dz_remainders what that leaves goes
        through them too, at 2.5 times the time of a large layer."""
        return self._dense_backward(dy, x, weight, None, activation, preact, x_activation, x_preact, need_dx, dx,
                                    dweight, dbias, dz_remainders)

    def grouped_linear_backward(self, dy, x, weight, offsets, activation="none", preact=None, x_activation="none",
                                x_preact=None, need_dx=True, dx=None, dweight=None, dbias=None, dz_remainders=False):
        """linear_backward of grouped_linear; dweight and dbias of a group
        without rows are zero."""
        if offsets is None:
            raise ValueError("offsets is missing")
        return self._dense_backward(dy, x, weight, offsets, activation, preact, x_activation, x_preact, need_dx, dx,
                                    dweight, dbias, dz_remainders)

    def adamw(self, params, grads, **how) -> AdamW:
        """An optimizer of these tensors (AdamW's arguments)."""
        return AdamW(self, params, grads, **how)

    def synchronize(self):
        B.painn_synchronize(self.ctx)

    def close(self):
        if self.ctx:
            B.painn_destroy(self.ctx)
            self.ctx = 0
