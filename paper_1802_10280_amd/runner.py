"""Per-layer driver used by the bench, the smoke check and the tests: packs the CSR once,
uploads it, owns the torch device buffers and issues the library calls of one forward pass.
It only marshals arguments; every step of the path runs inside libescoin.so.
FeedForwardRunner does the same for a feed-forward block of pruned linear layers."""
from __future__ import annotations

import numpy as np

from . import binding as B


class LayerRunner:
    def __init__(self, layer, path: str = "auto", flags: int = 0, stream=None, tuning=None, d_in=None):
        """d_in: a device tensor to read the input from instead of uploading the layer's own
        (the previous layer's output when layers are chained)."""
        import torch
        self.layer, self.flags, self.stream = layer, flags, stream
        s = layer.spec
        self.desc = B.desc_of(s)
        self.stretched = B.escoin_sconv_pack(self.desc, layer.rowptr, layer.colidx)
        dev = "cuda"
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)
        nz = layer.nnz > 0
        self.d_rowptr = up(layer.rowptr)
        self.d_colidx = up(self.stretched) if nz else torch.zeros(1, dtype=torch.int32, device=dev)
        self.d_value = up(layer.value) if nz else torch.zeros(1, dtype=torch.float32, device=dev)
        self.d_bias = up(layer.bias) if layer.bias is not None else None
        if d_in is not None:
            assert tuple(d_in.shape) == (s.N, s.C, s.H, s.W) and d_in.dtype == torch.float32
            self.d_in = d_in
        else:
            self.d_in = up(layer.input)
        self.d_padded = torch.empty(B.escoin_padded_elems(self.desc), dtype=torch.float32, device=dev)
        self.d_out = torch.empty((s.N, s.M, s.E, s.F), dtype=torch.float32, device=dev)
        self.path = "tiled" if path == "auto" else path
        if self.path == "tiled":
            if isinstance(tuning, dict):
                tuning = B.make_tuning(**tuning)
            self.plan = B.escoin_sconv_plan_build(self.desc, layer.rowptr, self.stretched,
                                                  layer.value, tuning)
            self.plan_info = B.plan_header(self.plan)
            self.d_plan = up(self.plan)
        elif self.path != "direct":
            raise ValueError(f"unknown sconv path {path!r}")

    @staticmethod
    def available_paths(layer):
        return ["tiled", "direct"]

    # -- one forward pass ---------------------------------------------------------------
    def pad_in(self):
        B.escoin_pad_in(self.desc, self.d_in, self.d_padded, self.stream)

    def sconv(self):
        B.escoin_sconv_forward(self.desc, self.d_rowptr, self.d_colidx, self.d_value,
                               self.d_padded, self.d_out, self.d_bias, self.flags, self.stream)

    def sconv_tiled(self):
        B.escoin_sconv_forward_tiled(self.desc, self.plan, self.d_plan, self.d_in, self.d_out,
                                     self.d_bias, self.flags, self.stream)

    def kernels(self):
        """The library calls of one forward pass, in order (the tiled path pads while staging,
        so it has no separate pad_in)."""
        return [self.sconv_tiled] if self.path == "tiled" else [self.pad_in, self.sconv]

    def kernel_names(self):
        return ["sconv"] if self.path == "tiled" else ["pad_in", "sconv"]

    def sconv_kernel_name(self):
        if self.path == "tiled":
            k = B.escoin_sconv_tiled_kernel(self.desc, self.plan) if self.d_plan.data_ptr() % 16 == 0 else 0
            if k:
                return "sconv_mfma_kernel" if k == 1 else f"sconv_pair_kernel<{k // 100}, {k // 10 % 10}, {k % 10}>"
            h = self.plan_info
            vw = h["VW"] if self.d_in.data_ptr() % 16 == 0 else 1
            if vw == 4 and h["n_dma"] > 0 and h["WW"] == 4:
                vw = 16       # staged by global -> LDS copies
            return f"sconv_tiled_kernel<{h['K']}, {h['Q']}, {h['B']}, {vw}>"
        return "sconv_direct_kernel"

    def run(self):
        for k in self.kernels():
            k()
        return self.d_out


TYPES = {"f32": B.T_F32, "f16": B.T_F16, "bf16": B.T_BF16}


class FeedForwardRunner:
    """One pruned feed-forward block: n = norm(x); g = silu(n Wg) * (n Wu); d = g Wd; h = x + gate * norm(d); and the next
    block's n = norm(h).  It owns the buffers of one number of tokens, and its plans; a program that has calls of several lengths makes
    one plan for the longest, and calls the library with the length of each."""

    def __init__(self, block, stream=None, before=None, eps: float = 1e-5):
        """before: the runner of the block before this one, whose h and n this one reads (they need no norm of their own)."""
        import torch
        self.block, self.stream, self.before = block, stream, before
        s = block.spec
        type, dt = TYPES[s.type], (torch.float32, torch.float16, torch.bfloat16)[TYPES[s.type]]
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to("cuda").to(dt)
        new = lambda width: torch.empty((s.T, width), dtype=dt, device="cuda")
        self.d_x, self.d_n = (before.d_h, before.d_next) if before is not None else (up(block.x), new(s.D))
        assert tuple(self.d_x.shape) == (s.T, s.D) and self.d_x.dtype == dt
        self.d_g, self.d_d, self.d_h, self.d_next = new(s.F), new(s.D), new(s.D), new(s.D)
        self.d_norm, self.d_post, self.d_pre, self.d_gate = (up(a) for a in (block.norm, block.post_norm, block.next_norm, block.gate))
        self.up_desc, self.down_desc = B.make_linear_desc(s.T, s.D, s.F, type, gated=True), B.make_linear_desc(s.T, s.F, s.D, type)
        self.up_plan = B.escoin_linear_plan_build(self.up_desc, *block.up)
        self.down_plan = B.escoin_linear_plan_build(self.down_desc, *block.down)
        self.d_up, self.d_down = (torch.from_numpy(p).to("cuda") for p in (self.up_plan, self.down_plan))
        self.first_desc = B.make_norm_desc(s.T, s.D, type, B.NORM_NONE, B.NORM_RMS, eps=eps)
        self.last_desc = B.make_norm_desc(s.T, s.D, type, B.NORM_RMS, B.NORM_RMS, eps=eps)

    def norm(self):
        B.escoin_norm_forward(self.first_desc, self.d_x, None, self.d_n, d_pre_weight=self.d_norm, stream=self.stream)

    def up(self):
        B.escoin_linear_forward(self.up_desc, self.up_plan, self.d_up, self.d_n, self.d_g, flags=B.F_SILU, stream=self.stream)

    def down(self):
        B.escoin_linear_forward(self.down_desc, self.down_plan, self.d_down, self.d_g, self.d_d, stream=self.stream)

    def sum(self):
        B.escoin_norm_forward(self.last_desc, self.d_x, self.d_h, self.d_next, d_y=self.d_d, d_gate=self.d_gate,
                              d_post_weight=self.d_post, d_pre_weight=self.d_pre, stream=self.stream)

    def kernels(self):
        """The library calls of one forward pass, in order."""
        return [*([self.norm] if self.before is None else []), self.up, self.down, self.sum]

    def kernel_names(self):
        return [k.__name__ for k in self.kernels()]

    def run(self):
        for k in self.kernels():
            k()
        return self.d_h, self.d_next
