"""Fitting gated efficiency heads to measured kernels (Sec. 5.3: per-family heads
learn log eta from dimensionless features).

    rows = feature_rows_of(inputs)            # ks_features: one row per (record, spec)
    data = Measurements(rows.x, rows.fam_off, measured_time / rows.t_roof)
    fit = GatedFit(in_dim=16, hidden=64)
    for _ in range(steps):
        loss = fit.step(data)                 # device tensor [NFAM]; nothing waits
    abi.ks_eval_steps(..., fit.heads, ...)    # the fitted heads price records

A step is ks_gated_loss (loss and gradients) and ks_adamw (all tensors in one
launch); it allocates nothing and can be captured into a graph.  A step is argument
marshalling, as in ``abi``: its arithmetic is in libks.so.  (``heads_for`` forms what a
category's learned columns add to its heads in torch, once for fitted heads.)

Rows measured on different devices (library versions, element types) carry a category
each, whose learned columns stand beside their 16 features:

    data = Measurements(rows.x, rows.fam_off, eta, ids=device_of_row, categories=8)
    fit = GatedFit(categories=8, dropout=0.1)
    ...
    abi.ks_eval_steps(..., fit.heads_for(3), ...)   # kernels of device 3
    abi.ks_eval_steps(..., fit.heads_for(None), ...)   # of a device never measured

A step is then ks_embed, ks_gated_forward, ks_eta_loss, ks_gated_backward, ks_embed_backward
and ks_adamw.  Dropout (of learned columns; of features: ``feature_dropout``) draws anew in
every step, in replays of a captured one too."""
from __future__ import annotations

import weakref
from types import SimpleNamespace

from . import abi


def feature_rows_of(inputs: abi.DeviceInputs, in_dim: int = 16, precision: str = "f32") -> SimpleNamespace:
    """The feature rows of every (record, spec) pair of ``inputs``: x
    [pairs][in_dim], t_roof [pairs], fam_off (of the pairs, family-major; within a
    family spec by spec)."""
    import torch
    n, s = inputs.desc.n_rows, inputs.n_specs
    dev = inputs.ws.device
    x = torch.empty((n * s, in_dim), dtype=torch.bfloat16 if precision == "bf16" else torch.float32, device=dev)
    roof = torch.empty(n * s, device=dev)
    with torch.cuda.device(dev):
        abi.ks_features(inputs.desc, inputs.specs_ptr, s, in_dim, abi.KS_BF16 if precision == "bf16" else abi.KS_F32,
                        x.data_ptr() if n else None, in_dim, roof.data_ptr() if n else None, inputs.ws_ptr,
                        inputs.ws_bytes, abi.current_stream())
    return SimpleNamespace(x=x, t_roof=roof, fam_off=[s * int(v) for v in inputs.desc.fam_off])


FEATURES = 16     # before the learned columns, which are as many


class Measurements:
    """Feature rows with their measured eta (NaN: never measured) and weights
    (None: 1 each), kept on the device.  ids: an int32 category below ``categories`` for
    each row of 16 features (others, as -1: none).  x is then a copy whose columns behind the
    features are the learned ones, written by each step, and the ids' order is found once:
    one fit at a time steps on such rows.  (Without ids several may, each on a stream or in
    a graph of its own.)"""

    def __init__(self, x, fam_off, eta, weight=None, huber: float = float("inf"), ids=None, categories: int = 0):
        import torch
        if eta.shape != x.shape[:1]:
            raise ValueError(f"eta is {tuple(eta.shape)}, not one per row of {tuple(x.shape)}")
        if any(t is not None and t.device != x.device for t in (eta, weight, ids)):
            raise ValueError("x, eta, weight and ids are not on one device")
        self.ids, self.categories = ids, 0
        self.noisy = None   # the rows that the last step which drops features has written
        if ids is not None:
            if ids.dtype != torch.int32 or ids.shape != eta.shape or not ids.is_contiguous():
                raise ValueError(f"ids are {ids.dtype} {tuple(ids.shape)}, not int32 {tuple(eta.shape)}")
            if x.shape[1] != FEATURES or categories < 1:
                raise ValueError(f"rows of {x.shape[1]} features with {categories} categories: {FEATURES} and at least one")
            self.categories = categories
            x = torch.cat([x, torch.zeros_like(x)], 1)
        self.x, self.eta, self.weight = x, eta, weight
        self.rows = abi.feature_rows(x, fam_off)
        self.target = abi.eta_target(eta, weight, huber)
        if ids is not None:
            self._learned(fam_off)
            self.sort()

    def _learned(self, fam_off):
        """What a step with learned columns writes and works in."""
        import torch

        def room(need):
            return torch.empty(need, dtype=torch.uint8, device=self.x.device)
        self.columns = abi.matrix(self.x[:, FEATURES:])
        self.fam_off = abi.family_offsets(fam_off)
        self.dz, self.dx = torch.empty_like(self.eta), torch.empty_like(self.x)
        self.rows_grad, self.columns_grad = abi.gated_grad(x=self.dx), abi.matrix(self.dx[:, FEATURES:])
        self.order = abi.id_order(len(self.eta), self.categories, self.x.device)
        self.sort_ws = room(abi.ks_embed_sort_workspace_bytes(self.order))
        self.back_ws = room(abi.ks_embed_backward_workspace_bytes(self.order, self.columns_grad))
        self.loss_ws = room(abi.ks_eta_loss_workspace_bytes(self.fam_off))

    def sort(self):
        """The order of the ids; to be called again when they have changed."""
        import torch
        with torch.cuda.device(self.x.device):
            abi.ks_embed_sort(self.ids.data_ptr(), self.order, self.sort_ws.data_ptr(), self.sort_ws.numel(),
                              abi.current_stream())

    def noise(self):
        """Rows for one fit that drops features: theirs but the constant one are written by
        each step."""
        x, features = self.x.clone(), FEATURES - 1
        return SimpleNamespace(x=x, rows=abi.feature_rows(x, list(self.rows.fam_off)),
                               columns=abi.matrix(x[:, FEATURES:]) if self.categories else None,
                               pair=(abi.matrix(self.x[:, :features]), abi.matrix(x[:, :features])))


class GatedFit:
    """Gated heads under AdamW: fp32 parameters, states of ``state_bits`` (32 or 8),
    and for precision "bf16" the bf16 copies that the heads read.  categories: how many
    there are learned columns for (0: none; else in_dim is 32); dropout: of their
    elements, feature_dropout: of the features but the constant one (not with in_dim 32
    and no categories: no dropout keeps both a feature's expected value and its square's)."""

    def __init__(self, in_dim: int = 16, hidden: int = 64, precision: str = "f32", seed: int = 0, lr: float = 3e-3,
                 weight_decay: float = 0.0, state_bits: int = 32, device="cuda", categories: int = 0, dropout: float = 0.0,
                 feature_dropout: float = 0.0):
        import torch
        if categories < 0 or (dropout and not categories):
            raise ValueError(f"{categories} categories, dropout of learned columns {dropout}")
        if not (0.0 <= dropout < 1.0 and 0.0 <= feature_dropout < 1.0):
            raise ValueError(f"dropout {dropout} or feature_dropout {feature_dropout} outside [0, 1)")
        if feature_dropout and in_dim != FEATURES and not categories:
            raise ValueError(f"feature_dropout of {in_dim} inputs: features would be dropped without their squares")
        in_dim = 2 * FEATURES if categories else in_dim
        g = torch.Generator().manual_seed(seed)
        n = abi.NFAM
        # gates and ups of order 1 for features of order 1; b3 = 0 puts eta at 2
        self.param = {"w1": torch.randn(n, hidden, in_dim, generator=g) * (2.0 / in_dim) ** 0.5,
                      "w2": torch.randn(n, hidden, in_dim, generator=g) * (2.0 / in_dim) ** 0.5,
                      "w3": torch.randn(n, hidden, generator=g) * (1.0 / hidden) ** 0.5,
                      "b3": torch.zeros(n)}
        if categories:   # (small: at first the rows differ by their features)
            self.param["table"] = torch.randn(categories, FEATURES, generator=g) * 0.1
        self.param = {k: v.to(device) for k, v in self.param.items()}
        low = precision == "bf16"
        self.weights = {k: v.bfloat16() if low else v for k, v in self.param.items()}
        self.block = abi.gated_heads(*(self.weights[k] for k in ("w1", "w2", "w3", "b3")))
        self.grad = {k: torch.zeros_like(v) for k, v in self.param.items()}
        self.loss = torch.zeros(n, device=device)
        self.count = torch.zeros(1, dtype=torch.int32, device=device)
        self.grad_struct = abi.gated_grad(**{k: self.grad[k] for k in ("w1", "w2", "w3", "b3")})
        self.drop = abi.drop(dropout, seed, 1, step_dev=self.count) if dropout else None
        self.feature_drop = abi.drop(feature_dropout, seed, 0, step_dev=self.count) if feature_dropout else None
        if categories:
            self.table, self.table_grad = abi.matrix(self.weights["table"]), abi.matrix(self.grad["table"])
        self.categories = categories
        self.state = {}
        tensors = []
        for k, v in self.param.items():
            st = {}
            if state_bits == 8:
                blocks = -(-v.numel() // 64)
                st = {"m": torch.zeros(v.shape, device=device).to(torch.float8_e4m3fn),
                      "v": torch.zeros(v.shape, device=device).to(torch.float8_e5m2),
                      "m_exp": torch.ones(blocks, dtype=torch.uint8, device=device),
                      "v_exp": torch.ones(blocks, dtype=torch.uint8, device=device)}
            else:
                st = {"m": torch.zeros_like(v), "v": torch.zeros_like(v)}
            self.state[k] = st
            tensors.append({"param": v, "grad": self.grad[k], **st, "copy": self.weights[k] if low else None,
                            "weight_decay": weight_decay if k in ("w1", "w2") else 0.0})
        self.tensors = abi.adamw_tensors(tensors)
        self.config = abi.adamw_config(lr, state_bits=state_bits, step_dev=self.count)
        self.ws, self.rooms = None, []
        self.noise = weakref.WeakKeyDictionary()   # Measurements -> the rows to drop features in

    @property
    def heads(self) -> abi.ks_heads:
        """The heads for the evaluation (of a fit with categories: ``heads_for``, since what
        the evaluation puts beside 16 features is their squares)."""
        if self.categories:
            raise ValueError("a fit with categories: heads_for(category)")
        return self.block

    def workspace(self, data: Measurements) -> int:
        """Room for a step on these rows; called by ``step``, and before a capture (of a fit
        that drops features on the steps' stream, or one that it waits for: a copy of the rows
        is made).  Smaller rooms are kept: captured steps go on using them."""
        import torch
        like = self.weights["w1"]
        if data.x.device != like.device or data.x.dtype != like.dtype or data.x.shape[1] != self.block.in_dim:
            raise ValueError(f"rows are {data.x.dtype} [{data.x.shape[1]}] on {data.x.device}, "
                             f"not {like.dtype} [{self.block.in_dim}] on {like.device}")
        if data.categories != self.categories:
            raise ValueError(f"rows of {data.categories} categories for a fit of {self.categories}")
        need = abi.ks_gated_workspace_bytes(self.block, data.rows)
        if need == 0:
            raise abi.KsError(abi.KS_EINVAL, abi.ks_last_error())
        new = self.feature_drop is not None and data not in self.noise
        if new and data.x.is_cuda:
            with torch.cuda.device(data.x.device):
                if torch.cuda.is_current_stream_capturing():   # (eager steps would lack the copy until a replay)
                    raise RuntimeError("a fit that drops features: workspace(rows) before a capture")
        if self.ws is None or self.ws.numel() < need:
            self.ws = torch.empty(need, dtype=torch.uint8, device=self.loss.device)
            self.rooms.append(self.ws)
        if self.feature_drop is not None:
            if new:
                self.noise[data] = data.noise()
            data.noisy = self.noise[data].x
        return need

    def gradients(self, data: Measurements):
        """The loss per family [NFAM] and, in ``self.grad``, its gradients; the next
        call writes the same tensors."""
        import torch
        need = self.workspace(data)
        with torch.cuda.device(self.loss.device):
            s, ws = abi.current_stream(), self.ws.data_ptr()
            noise = None if self.feature_drop is None else self.noise[data]
            rows = data.rows if noise is None else noise.rows
            if noise is not None:
                abi.ks_dropout(self.feature_drop, *noise.pair, s)
            if not self.categories:
                abi.ks_gated_loss(self.block, rows, data.target, self.loss.data_ptr(), None, self.grad_struct, ws, need, s)
                return self.loss
            columns, dz = data.columns if noise is None else noise.columns, data.dz.data_ptr()
            abi.ks_embed(self.table, 1.0, data.ids.data_ptr(), self.drop, columns, s)
            abi.ks_gated_forward(self.block, rows, dz, s)
            abi.ks_eta_loss(data.fam_off, dz, data.target, self.loss.data_ptr(), dz, data.loss_ws.data_ptr(),
                            data.loss_ws.numel(), s)
            abi.ks_gated_backward(self.block, rows, dz, self.grad_struct, ws, need, s)
            abi.ks_gated_backward(self.block, rows, dz, data.rows_grad, ws, need, s)
            abi.ks_embed_backward(data.order, 1.0, data.columns_grad, self.drop, self.table_grad, data.back_ws.data_ptr(),
                                  data.back_ws.numel(), s)
        return self.loss

    def step(self, data: Measurements):
        """One step; returns the loss per family before it (``gradients``)."""
        import torch
        loss = self.gradients(data)
        with torch.cuda.device(loss.device):
            abi.ks_adamw(self.config, self.tensors, abi.current_stream())
        return loss

    def heads_for(self, category: int | None = None, bounded=None, grid=None) -> abi.ks_heads:
        """Heads of 16 features for one category (None: its learned columns are 0, as for
        rows without one): feature 15 is 1, so what the learned columns e add to gates and
        ups, W[:, 16:] e, goes to their column 15: formed in fp32, for bf16 heads rounded once
        more, as those are bf16 throughout.  The weights as of now, in tensors that stay with
        the struct (``weights``); bounded, grid: as for ``abi.gated_heads``."""
        if not self.categories:
            raise ValueError("a fit without categories: its heads are ``heads``")
        if category is not None and not 0 <= category < self.categories:
            raise ValueError(f"category {category} outside 0 .. {self.categories - 1}")
        w = {k: self.weights[k].float() for k in ("w1", "w2")}
        out = {k: v[:, :, :FEATURES].clone() for k, v in w.items()}
        if category is not None:
            e = self.weights["table"][category].float()
            for k, v in w.items():
                out[k][:, :, FEATURES - 1] += (v[:, :, FEATURES:] * e).sum(-1)
        like = self.weights["w3"]
        out = {k: v.to(like.dtype) for k, v in out.items()} | {k: self.weights[k].clone() for k in ("w3", "b3")}
        heads = abi.gated_heads(out["w1"], out["w2"], out["w3"], out["b3"], bounded, grid)
        heads.weights = out
        return heads
