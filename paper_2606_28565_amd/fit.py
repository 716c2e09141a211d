"""Fitting gated efficiency heads to measured kernels (Sec. 5.3: per-family heads
learn log eta from dimensionless features).

    rows = feature_rows_of(inputs)            # ks_features: one row per (record, spec)
    data = Measurements(rows.x, rows.fam_off, measured_time / rows.t_roof)
    fit = GatedFit(in_dim=16, hidden=64)
    for _ in range(steps):
        loss = fit.step(data)                 # device tensor [NFAM]; nothing waits
    abi.ks_eval_steps(..., fit.heads, ...)    # the fitted heads price records

A step is ks_gated_loss (loss and gradients) and ks_adamw (all tensors in one
launch); it allocates nothing and can be captured into a graph.  Argument
marshalling only, as in ``abi``: the arithmetic is in libks.so."""
from __future__ import annotations

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


class Measurements:
    """Feature rows with their measured eta (NaN: never measured) and weights
    (None: 1 each), kept on the device."""

    def __init__(self, x, fam_off, eta, weight=None, huber: float = float("inf")):
        if eta.shape != x.shape[:1]:
            raise ValueError(f"eta is {tuple(eta.shape)}, not one per row of {tuple(x.shape)}")
        if any(t is not None and t.device != x.device for t in (eta, weight)):
            raise ValueError("x, eta and weight are not on one device")
        self.x, self.eta, self.weight = x, eta, weight
        self.rows = abi.feature_rows(x, fam_off)
        self.target = abi.eta_target(eta, weight, huber)


class GatedFit:
    """Gated heads under AdamW: fp32 parameters, states of ``state_bits`` (32 or 8),
    and for precision "bf16" the bf16 copies that the heads read."""

    def __init__(self, in_dim: int = 16, hidden: int = 64, precision: str = "f32", seed: int = 0, lr: float = 3e-3,
                 weight_decay: float = 0.0, state_bits: int = 32, device="cuda"):
        import torch
        g = torch.Generator().manual_seed(seed)
        n = abi.NFAM
        # gates and ups of order 1 for features of order 1; b3 = 0 puts eta at 2
        self.param = {"w1": torch.randn(n, hidden, in_dim, generator=g) * (2.0 / in_dim) ** 0.5,
                      "w2": torch.randn(n, hidden, in_dim, generator=g) * (2.0 / in_dim) ** 0.5,
                      "w3": torch.randn(n, hidden, generator=g) * (1.0 / hidden) ** 0.5,
                      "b3": torch.zeros(n)}
        self.param = {k: v.to(device) for k, v in self.param.items()}
        low = precision == "bf16"
        self.weights = {k: v.bfloat16() if low else v for k, v in self.param.items()}
        self.heads = abi.gated_heads(*(self.weights[k] for k in ("w1", "w2", "w3", "b3")))
        self.grad = {k: torch.zeros_like(v) for k, v in self.param.items()}
        self.grad_struct = abi.gated_grad(**self.grad)
        self.loss = torch.zeros(n, device=device)
        self.count = torch.zeros(1, dtype=torch.int32, device=device)
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

    def workspace(self, data: Measurements) -> int:
        """Room for a step on these rows; called by ``step``, and before a capture.
        Smaller rooms are kept: captured steps go on using them."""
        import torch
        like = self.weights["w1"]
        if data.x.device != like.device or data.x.dtype != like.dtype or data.x.shape[1] != self.heads.in_dim:
            raise ValueError(f"rows are {data.x.dtype} [{data.x.shape[1]}] on {data.x.device}, "
                             f"not {like.dtype} [{self.heads.in_dim}] on {like.device}")
        need = abi.ks_gated_workspace_bytes(self.heads, data.rows)
        if need == 0:
            raise abi.KsError(abi.KS_EINVAL, abi.ks_last_error())
        if self.ws is None or self.ws.numel() < need:
            self.ws = torch.empty(need, dtype=torch.uint8, device=self.loss.device)
            self.rooms.append(self.ws)
        return need

    def gradients(self, data: Measurements):
        """The loss per family [NFAM] and, in ``self.grad``, its gradients; the next
        call writes the same tensors."""
        import torch
        need = self.workspace(data)
        with torch.cuda.device(self.loss.device):
            abi.ks_gated_loss(self.heads, data.rows, data.target, self.loss.data_ptr(), None, self.grad_struct,
                              self.ws.data_ptr(), need, abi.current_stream())
        return self.loss

    def step(self, data: Measurements):
        """One step; returns the loss per family before it (``gradients``)."""
        import torch
        loss = self.gradients(data)
        with torch.cuda.device(loss.device):
            abi.ks_adamw(self.config, self.tensors, abi.current_stream())
        return loss
