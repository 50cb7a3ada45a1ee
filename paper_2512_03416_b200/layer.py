"""The decoder layer around the attention step (ts_layer_*), with PyTorch supplying device memory
and the stream. All computation happens inside libtokenscale.so; this file only marshals arguments.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding as B
from .decoder import Decoder, TsError, _check


class DecoderLayer:
    """RMSNorm, fused QKV projection with rotary embedding, the decoder's paged attention step,
    output projection and gated MLP, bound to a Decoder (its pool, block tables and counters).

    Weights are int16 CUDA tensors holding bf16 bit patterns, [out features, in features]:
    w_norm1 [hidden], w_qkv [(Hq + 2 Hkv) D, hidden], w_o [hidden, Hq D], w_norm2 [hidden],
    w_gate, w_up [intermediate, hidden], w_down [hidden, intermediate]."""

    def __init__(self, dec: Decoder, w_norm1, w_qkv, w_o, w_norm2, w_gate, w_up, w_down, max_position: int,
                 rms_eps: float = 0.0, rope_theta: float = 0.0):
        self.dec = dec
        hidden = int(w_norm1.numel())
        inter = int(w_gate.shape[0])
        stream = torch.cuda.current_stream(dec.device).cuda_stream
        self.w_gate_up = torch.empty((2 * inter, hidden), dtype=torch.int16, device=dec.device)
        _check(B.ts_pack_gate_up(w_gate.data_ptr(), w_up.data_ptr(), self.w_gate_up.data_ptr(), inter, hidden, stream),
               "ts_pack_gate_up")
        self.weights = (w_norm1, w_qkv, w_o, w_norm2, w_down)          # keep the caller's tensors alive
        cfg = B.ts_layer_config(hidden, inter, max_position, rms_eps, rope_theta, w_norm1.data_ptr(), w_qkv.data_ptr(),
                                w_o.data_ptr(), w_norm2.data_ptr(), self.w_gate_up.data_ptr(), w_down.data_ptr(), None, 0)
        nbytes = B.ts_layer_workspace_bytes(dec.cfg, cfg)
        if nbytes == 0:
            raise TsError(B.TS_ERR_UNSUPPORTED, "ts_layer_workspace_bytes")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=dec.device)
        cfg.workspace, cfg.workspace_bytes = self.workspace.data_ptr(), nbytes
        self.cfg = cfg
        rc, self.handle = B.ts_layer_create(dec.ctx, cfg, stream)
        _check(rc, "ts_layer_create")

    def set_adapters(self, qkv=None, o=None, gate_up=None, down=None) -> None:
        """Adapters (adapters.Adapters, one count for all) of the projections; b of gate_up in the packed order (pack_gate_up_adapters).
        Without any: none. Synchronises, since earlier steps may still use the former ones."""
        torch.cuda.synchronize(self.dec.device)
        given = dict(qkv=qkv, o=o, gate_up=gate_up, down=down)
        width = self.weights[1].shape[0], self.weights[1].shape[1], self.weights[2].shape[1], self.w_gate_up.shape[0], self.weights[4].shape[1]
        shapes = dict(qkv=(width[0], width[1]), o=(width[1], width[2]), gate_up=(width[3], width[1]), down=(width[1], width[4]))
        for name, ad in given.items():
            if ad is not None and ((ad.n, ad.k) != shapes[name] or ad.device != self.dec.device):
                raise ValueError(f"the adapters of {name} must be of a projection {list(shapes[name])} on {self.dec.device}")
            if ad is not None and ad.rows != (name if name in ("qkv", "gate_up") else "plain"):
                raise ValueError(f"the adapters of {name} are laid out for rows={ad.rows!r}")
        args = B.ts_layer_adapters(*[None if ad is None else ctypes.pointer(ad.args) for ad in given.values()], None, 0)
        workspace = None
        if any(ad is not None for ad in given.values()):
            nbytes = B.ts_layer_adapters_workspace_bytes(self.dec.cfg, args)
            if nbytes == 0:
                raise TsError(B.TS_ERR_UNSUPPORTED, "ts_layer_adapters_workspace_bytes")
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.dec.device)
            args.workspace, args.workspace_bytes = workspace.data_ptr(), nbytes
        _check(B.ts_layer_attach_adapters(self.handle, args), "ts_layer_attach_adapters")
        self.adapters = (given, workspace)                             # kept alive

    def pack_gate_up_adapters(self, b_gate, b_up) -> torch.Tensor:
        """b of gate_up [adapters, 2 intermediate, rank] from those of gate and up [adapters, intermediate, rank] of one rank (their rows
        in the order of the packed weights)."""
        for t, what in ((b_gate, "b_gate"), (b_up, "b_up")):
            if t.dim() != 3 or t.dtype not in (torch.bfloat16, torch.int16, torch.uint16) or t.device != self.dec.device:
                raise ValueError(f"{what} must be a bf16 (or int16, uint16) tensor [adapters, intermediate, rank] on {self.dec.device}")
        if b_gate.shape != b_up.shape or b_gate.dtype != b_up.dtype:
            raise ValueError(f"b_gate and b_up must be of one shape and type, not {list(b_gate.shape)} {b_gate.dtype} and {list(b_up.shape)} {b_up.dtype}")
        n, inter, rank = b_gate.shape
        b_gate, b_up = b_gate.contiguous(), b_up.contiguous()
        out = torch.empty((n, 2 * inter, rank), dtype=b_gate.dtype, device=self.dec.device)
        with torch.cuda.device(self.dec.device):
            for i in range(n):
                _check(B.ts_pack_gate_up(b_gate[i].data_ptr(), b_up[i].data_ptr(), out[i].data_ptr(), inter, rank, self.dec._stream()),
                       "ts_pack_gate_up")
        return out

    def close(self) -> None:
        if getattr(self, "handle", None):
            torch.cuda.synchronize(self.dec.device)
            B.ts_layer_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def make_step(self, slots, q_len, ctx_len, keep_len: bool = False):
        return B.make_step(slots, q_len, ctx_len, 0, 0, 0, 0, B.TS_STEP_KEEP_LEN if keep_len else 0)

    def step_prepared(self, st, x_in, x_out, adapters=None) -> None:
        """adapters: per row of the step the adapter it uses (-1: none); None: no adapters."""
        if adapters is None:
            _check(B.ts_layer_step(self.handle, st, x_in.data_ptr(), x_out.data_ptr(),
                                   self.dec._stream()), "ts_layer_step")
            return
        if len(adapters) != st.n_rows:
            raise ValueError("one adapter (or -1) per row of the step")
        _check(B.ts_layer_step_adapted(self.handle, st, adapters, x_in.data_ptr(), x_out.data_ptr(),
                                       self.dec._stream()), "ts_layer_step_adapted")

    def step(self, slots, q_len, ctx_len, x_in, x_out, keep_len: bool = False, adapters=None) -> None:
        st, _keep = self.make_step(slots, q_len, ctx_len, keep_len)
        self.step_prepared(st, x_in, x_out, adapters)
