"""Convenience wrapper around the C-ABI calls for one fixed layer layout: owns the device-side
descriptor tables, the workspace and the stream buffers, and strings the entry points together
(fit codes -> encode -> decode-aggregate).  Orchestration only; all arithmetic is in libco3.so.
"""
from __future__ import annotations

import numpy as np
import torch

from . import binding as B


class Co3Session:
    def __init__(self, sizes, fmts, n_clients: int, decay: float, device="cuda"):
        """sizes: elements per layer; fmts: (exp_bits, mant_bits, flags, scale, inv_scale) per layer."""
        self.sizes = [int(n) for n in sizes]
        self.n_seg = len(self.sizes)
        self.n_elem = int(sum(self.sizes))
        self.n_clients = int(n_clients)
        self.decay = float(decay)
        self.device = torch.device(device)
        self.fmts_host = B.make_fmts(fmts)
        self.fmts = B.to_device(self.fmts_host, self.device)
        self.segs = B.to_device(B.make_segs(self.sizes), self.device)
        self.codes_host = None
        self.codes = None
        self.stride = (self.n_elem + 3) // 4 * 4                      # keeps every client's vector 16-byte aligned
        ws_bytes = B.co3_workspace_bytes(self.n_elem, self.n_seg, self.n_clients)
        self.workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=self.device)
        self.capacity = B.co3_stream_capacity_bytes(self.n_elem, self.n_seg)
        self.streams = torch.empty(self.n_clients * self.capacity, dtype=torch.uint8, device=self.device)
        base = self.streams.data_ptr()
        self.stream_ptrs = torch.tensor([base + u * self.capacity for u in range(self.n_clients)],
                                        dtype=torch.int64, device=self.device)
        self.res_enc = torch.zeros(self.n_clients * B.RESULT_DTYPE.itemsize, dtype=torch.uint8, device=self.device)
        self.res_dec = torch.zeros(B.RESULT_DTYPE.itemsize, dtype=torch.uint8, device=self.device)
        self.res_fit = torch.zeros(B.RESULT_DTYPE.itemsize, dtype=torch.uint8, device=self.device)
        self.res_model = torch.zeros(B.RESULT_DTYPE.itemsize, dtype=torch.uint8, device=self.device)
        self.res_f8 = torch.zeros(B.RESULT_DTYPE.itemsize, dtype=torch.uint8, device=self.device)
        self.avg = torch.empty(self.n_elem, dtype=torch.float32, device=self.device)
        self.hist = torch.zeros(max(1, self.n_seg) * 256, dtype=torch.int64, device=self.device)

    # -- buffers ------------------------------------------------------------------------------
    def new_client_buffer(self, dtype=torch.float32) -> torch.Tensor:
        """Zeroed [n_clients * stride] buffer for gradients or memories."""
        return torch.zeros(self.n_clients * self.stride, dtype=dtype, device=self.device)

    def client_view(self, buf: torch.Tensor, u: int) -> torch.Tensor:
        return buf[u * self.stride:u * self.stride + self.n_elem]

    # -- multiplier fitting -------------------------------------------------------------------
    def fit_scales(self, grads: torch.Tensor, mems, log_tab: torch.Tensor, beta0: float, dbeta: float,
                   seg_tab=None, stats_out=None, stream=None) -> None:
        """Refits scale / inv_scale of every layer's format on the device from this round's gradients (and
        memories, if given): log_tab float32[n_tab][n_beta] and seg_tab int32[n_seg] (optional) are CUDA tensors.
        The host copy of the formats is stale afterwards until fmts_from_device() is called."""
        st = B.co3_fit_scale(grads, mems, self.decay, self.fmts, self.segs, self.n_seg, self.n_elem, self.n_clients,
                             self.stride, log_tab, seg_tab, log_tab.shape[0], log_tab.shape[1], beta0, dbeta,
                             stats_out, self.res_fit, self.workspace, stream)
        self._check(st, "co3_fit_scale")

    def error_magnitude(self, grads: torch.Tensor, mems: torch.Tensor, stream=None) -> torch.Tensor:
        """float64[n_clients][n_seg][2] on the device: l1 norm of each layer's gradient and memory per client."""
        out = torch.empty((self.n_clients, self.n_seg, 2), dtype=torch.float64, device=self.device)
        st = B.co3_error_magnitude(grads, mems, self.segs, self.n_seg, self.n_elem, self.n_clients, self.stride, out,
                                   self.res_fit, self.workspace, stream)
        self._check(st, "co3_error_magnitude")
        return out

    def fmts_from_device(self) -> np.ndarray:
        raw = self.fmts.cpu().numpy().tobytes()[:self.n_seg * B.FMT_DTYPE.itemsize]
        self.fmts_host = np.frombuffer(raw, dtype=B.FMT_DTYPE).copy()
        return self.fmts_host

    # -- code fitting -------------------------------------------------------------------------
    def histogram(self, grads: torch.Tensor, mems: torch.Tensor, stream=None, sym_out=None, to_host: bool = True):
        """Symbol counts per layer summed over clients for this round; `mems` is updated like a real round
        and, if `sym_out` is given, the symbols are kept for co3_encode_symbols.  The counts stay in
        self.hist on the device; to_host=False skips the copy to the host (and its synchronisation)."""
        st = B.co3_convert(grads, mems, self.decay, self.fmts, self.segs, self.n_seg, self.n_elem, self.n_clients,
                           self.stride, sym_out, self.hist, self.res_enc, self.workspace, stream)
        self._check(st, "co3_convert")
        if not to_host:
            return None
        return self.hist.cpu().numpy().astype(np.uint64).reshape(-1, 256)[:self.n_seg]

    def histogram_only(self, grads: torch.Tensor, mems: torch.Tensor, stream=None, to_host: bool = True):
        """The same counts without running the round: neither `mems` nor anything else is written."""
        st = B.co3_histogram(grads, mems, self.decay, self.fmts, self.segs, self.n_seg, self.n_elem, self.n_clients,
                             self.stride, self.hist, self.res_enc, self.workspace, stream)
        self._check(st, "co3_histogram")
        if not to_host:
            return None
        return self.hist.cpu().numpy().astype(np.uint64).reshape(-1, 256)[:self.n_seg]

    def set_codes_from_weights(self, weights: np.ndarray) -> None:
        """weights: uint64[n_seg][256] (histogram counts or model weights); one Huffman code per layer."""
        codes = np.zeros(self.n_seg, dtype=B.CODE_DTYPE)
        for k in range(self.n_seg):
            st, c = B.co3_code_build(weights[k], self.fmts_host[k:k + 1])
            self._check(st, "co3_code_build")
            codes[k] = c[0]
        self.set_codes(codes)

    def set_codes_from_histogram_device(self, stream=None) -> None:
        """One Huffman code per layer from the histogram the last histogram() call left on the device; the
        tables are built there too (the host copy of the codes is dropped)."""
        if self.codes is None:
            self.codes = torch.zeros(max(1, self.n_seg) * B.CODE_DTYPE.itemsize, dtype=torch.uint8, device=self.device)
        self.codes_host = None
        st = B.co3_code_build_device(self.hist, self.fmts, self.n_seg, self.codes, self.res_fit, stream)
        self._check(st, "co3_code_build_device")

    def set_codes_from_model_device(self, stats: torch.Tensor, stream=None) -> None:
        """One Huffman code per layer from the GenNorm model: `stats` is the float64[n_seg][4] tensor a fit_scales
        call filled (beta and alpha per layer); weights and tables are built on the device (self.hist then holds
        the model weights, not counts)."""
        st = B.co3_model_weights(self.fmts, stats, self.n_seg, self.hist, self.res_model, stream)
        self._check(st, "co3_model_weights")
        self.set_codes_from_histogram_device(stream)

    def set_codes(self, codes: np.ndarray) -> None:
        self.codes_host = codes
        self.codes = B.to_device(codes, self.device)

    # -- the two hot calls ---------------------------------------------------------------------
    def encode(self, grads: torch.Tensor, mems: torch.Tensor, stream=None) -> None:
        st = B.co3_encode(grads, mems, self.decay, self.fmts, self.codes, self.segs, self.n_seg, self.n_elem,
                          self.n_clients, self.stride, self.streams, self.capacity, self.workspace, self.res_enc,
                          stream=stream)
        self._check(st, "co3_encode")

    def encode_symbols(self, sym: torch.Tensor, stream=None) -> None:
        st = B.co3_encode_symbols(sym, self.codes, self.segs, self.n_seg, self.n_elem, self.n_clients, self.stride,
                                  self.streams, self.capacity, self.workspace, self.res_enc, stream=stream)
        self._check(st, "co3_encode_symbols")

    def decode_aggregate(self, stream=None) -> torch.Tensor:
        st = B.co3_decode_aggregate(self.stream_ptrs, self.capacity, self.n_clients, self.fmts, self.codes,
                                    self.segs, self.n_seg, self.n_elem, self.avg, self.workspace, self.res_dec,
                                    stream=stream)
        self._check(st, "co3_decode_aggregate")
        return self.avg

    def decode_aggregate_update(self, params: torch.Tensor, lr: float, want_avg: bool = False, stream=None):
        """Decode, average and apply params <- params - lr * avg in the same kernel."""
        st = B.co3_decode_aggregate_update(self.stream_ptrs, self.capacity, self.n_clients, self.fmts, self.codes,
                                           self.segs, self.n_seg, self.n_elem, lr, params,
                                           self.avg if want_avg else None, self.workspace, self.res_dec, stream=stream)
        self._check(st, "co3_decode_aggregate_update")
        return self.avg if want_avg else None

    # -- layer norm at the clients ---------------------------------------------------------------
    def new_layer_norm_workspace(self, rows: int, cols: int) -> torch.Tensor:
        """Workspace for layer_norm_backward with `rows` rows of each client."""
        return torch.empty(B.co3_layer_norm_workspace_bytes(rows, cols, self.n_clients), dtype=torch.uint8,
                           device=self.device)

    def layer_norm(self, x: torch.Tensor, params: torch.Tensor, gain: int, bias: int, y: torch.Tensor,
                   mean=None, rstd=None, eps: float = 1e-5, stream=None) -> None:
        """y <- layer norm of the rows of x with layers `gain` and `bias` of the parameter vector."""
        self._check_width(x, gain, bias)
        st = B.co3_layer_norm(x, self._layer(params, gain), self._layer(params, bias), y, mean, rstd, eps, stream)
        self._check(st, "co3_layer_norm")

    def layer_norm_backward(self, dy, x, params, gain: int, bias: int, mean, rstd, dx, grads, workspace,
                            accumulate: bool = False, stream=None) -> None:
        """Its gradients for the rows of all clients, client after client: dx, and every client's gradients of the two
        layers in its own vector of `grads`."""
        self._check_width(x, gain, bias)
        at = [sum(self.sizes[:k]) for k in (gain, bias)]
        st = B.co3_layer_norm_backward(dy, x, self._layer(params, gain), mean, rstd, dx, grads[at[0]:], grads[at[1]:],
                                       self.n_clients, self.stride, workspace, accumulate, stream)
        self._check(st, "co3_layer_norm_backward")

    # -- linear layers on 8-bit blocks at the clients ----------------------------------------------
    def new_f8(self, rows: int, cols: int, kind: int = B.F8_ROWS) -> torch.Tensor:
        """Room for a rows x cols matrix in 8-bit blocks."""
        return torch.empty(B.co3_f8_bytes(rows, cols, kind), dtype=torch.uint8, device=self.device)

    def new_linear_workspace(self, rows: int, outs: int, ins: int) -> torch.Tensor:
        """Workspace for linear_backward with `rows` rows of each client."""
        return torch.empty(B.co3_f8_weight_gradient_workspace_bytes(rows, outs, ins, self.n_clients), dtype=torch.uint8,
                           device=self.device)

    def pack_weights(self, params: torch.Tensor, weight: int, shape, w8: torch.Tensor, stream=None) -> None:
        """w8 (new_f8(*shape, F8_SQUARE)) <- layer `weight` of the parameter vector, (outputs, inputs) = shape."""
        st = B.co3_f8_pack(self._layer(params, weight).view(shape), w8, B.F8_SQUARE, stream)
        self._check(st, "co3_f8_pack")

    def linear(self, x, x8: torch.Tensor, w8: torch.Tensor, params: torch.Tensor, bias, y: torch.Tensor, cols=None, stream=None) -> None:
        """y <- x W^T + layer `bias` of the parameter vector (None: without); x is kept in x8 for linear_backward.  x None: x8
        holds the inputs (`cols` of them a row) already, from co3_f8_activation for instance."""
        b = None if bias is None else self._layer(params, bias)
        if b is not None and b.numel() != y.shape[1]:
            raise ValueError("layer %d is not of the outputs' length" % bias)
        st = B.co3_f8_linear(x, x8, w8, b, y, False, cols, self.res_f8, stream)
        self._check(st, "co3_f8_linear")

    def linear_backward(self, dy, dy8, x8, w8, weight: int, bias, shape, dx, grads, workspace, accumulate: bool = False, stream=None) -> None:
        """Gradients of `linear` for the rows of all clients, client after client: every client's gradients of layers `weight`
        and `bias` in its own vector of `grads`, and dx (None: not wanted; otherwise dy8 is room for dy in 8-bit blocks)."""
        outs, ins = shape
        if self.sizes[weight] != outs * ins or (bias is not None and self.sizes[bias] != outs) or dy.dim() != 2 or dy.shape[1] != outs:
            raise ValueError("layers and gradients are not of this shape")
        at = sum(self.sizes[:weight])
        db = None if bias is None else grads[sum(self.sizes[:bias]):]
        st = B.co3_f8_weight_gradient(dy, x8, ins, grads[at:], db, self.n_clients, self.stride, workspace, accumulate, self.res_f8, stream)
        self._check(st, "co3_f8_weight_gradient")
        if dx is not None:
            st = B.co3_f8_linear(dy, dy8, w8, None, dx, True, None, self.res_f8, stream)
            self._check(st, "co3_f8_linear")

    def f8_result(self) -> np.ndarray:
        """The last failure of the calls above, if any (cleared at the start of the session)."""
        return B.read_results(self.res_f8, 1)

    def _check_width(self, x: torch.Tensor, gain: int, bias: int) -> None:
        if x.dim() != 2 or x.shape[1] != self.sizes[gain] or x.shape[1] != self.sizes[bias]:
            raise ValueError("layers %d and %d are not of the rows' length" % (gain, bias))

    def _layer(self, vec: torch.Tensor, k: int) -> torch.Tensor:
        at = sum(self.sizes[:k])
        return vec[at:at + self.sizes[k]]

    # -- the orthogonalised step at the server ---------------------------------------------------
    def setup_muon(self, shapes, mu: float = 0.95, nesterov: bool = True, ns=None) -> None:
        """shapes[k]: (rows, cols) of layer k, or None where the momentum itself is the update (gains, biases).
        Matrices get the scale sqrt(max(1, rows / cols)), so that a step changes outputs alike at every shape."""
        mats, at = [], 0
        for n, shape in zip(self.sizes, shapes, strict=True):
            rows, cols = (1, n) if shape is None else shape
            if rows * cols != n:
                raise ValueError("a layer of %d elements is no %d x %d matrix" % (n, rows, cols))
            mats.append((at, rows, cols, cols, 1.0, B.MAT_PLAIN) if shape is None else
                        (at, rows, cols, cols, max(1.0, rows / max(cols, 1)) ** 0.5, 0))
            at += n
        self.mats = B.make_mats(mats)
        self.mu, self.nesterov, self.ns = float(mu), bool(nesterov), ns
        self.momentum = torch.zeros(self.n_elem, dtype=torch.float32, device=self.device)
        self.muon_workspace = torch.empty(B.co3_orthogonalize_workspace_bytes(self.mats), dtype=torch.uint8,
                                          device=self.device)
        self.res_muon = torch.zeros(B.RESULT_DTYPE.itemsize, dtype=torch.uint8, device=self.device)

    def muon_update(self, params: torch.Tensor, lr: float, weight_decay: float = 0.0, stream=None) -> None:
        """The server's step on the average that decode_aggregate left in self.avg (after setup_muon)."""
        st = B.co3_muon_update(self.avg, self.momentum, params, self.mats, self.mu, self.nesterov, lr, weight_decay,
                               self.muon_workspace, self.res_muon, self.ns, stream)
        self._check(st, "co3_muon_update")

    def muon_result(self) -> np.ndarray:
        return B.read_results(self.res_muon, 1)

    # -- results --------------------------------------------------------------------------------
    def encode_results(self) -> np.ndarray:
        return B.read_results(self.res_enc, self.n_clients)

    def fit_result(self) -> np.ndarray:
        return B.read_results(self.res_fit, 1)

    def model_result(self) -> np.ndarray:
        return B.read_results(self.res_model, 1)

    def decode_result(self) -> np.ndarray:
        return B.read_results(self.res_dec, 1)

    def stream_bytes(self, u: int) -> np.ndarray:
        used = int(self.encode_results()[u]["container_bytes"])
        return self.streams[u * self.capacity:u * self.capacity + used].cpu().numpy()

    @staticmethod
    def _check(st: int, what: str) -> None:
        if st != B.OK:
            raise RuntimeError("%s failed: %s" % (what, B.co3_status_string(st)))
