"""ctypes binding over libmoonwalk.so: argument marshalling only.

Every step of the Moonwalk path runs inside the CUDA library; this module converts Python
objects (torch tensors used purely as device buffers) into the pointers and sizes of the C ABI
declared in include/moonwalk.h.  There is no CPU fallback: if the library is missing or a CUDA
device is absent, calls raise.
"""
from __future__ import annotations

import array
import ctypes as C
import operator
import os
from typing import List, NamedTuple, Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmoonwalk.so")

MW_OK = 0
STATUS_NAMES = ["MW_OK", "MW_ERR_INVALID_ARG", "MW_ERR_UNSUPPORTED", "MW_ERR_WORKSPACE",
                "MW_ERR_STATE", "MW_ERR_NOT_SUBMERSIVE", "MW_ERR_TIMEOUT", "MW_ERR_CUDA"]
KIND = {"dense": 0, "conv2d": 1, "head": 2, "conv1d": 3}
ACT = {"none": 0, "leaky_relu": 1, "relu": 2}
PREC = {"f64": 0, "f32": 1, "bf16_f32acc": 2}
LOSS = {"half_sse": 0, "mse_mean": 1, "xent_mean": 2}
BACKEND = {"auto": 0, "simt": 1, "tensor": 2}


class MwError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        name = STATUS_NAMES[code] if 0 <= code < len(STATUS_NAMES) else str(code)
        super().__init__(f"{where}: {name}")


class LayerDesc(C.Structure):
    _fields_ = [("kind", C.c_int32), ("act", C.c_int32), ("slope", C.c_double),
                ("n_in", C.c_int32), ("n_out", C.c_int32), ("H", C.c_int32), ("W", C.c_int32),
                ("C_in", C.c_int32), ("C_out", C.c_int32), ("k", C.c_int32),
                ("stride", C.c_int32), ("pad", C.c_int32)]


class NetOpts(C.Structure):
    _fields_ = [("prec", C.c_int32), ("loss", C.c_int32), ("reseed_every", C.c_int32),
                ("conv_vijp_iters", C.c_int32), ("backend", C.c_int32),
                ("inverse_iters", C.c_int32), ("resident_inverse", C.c_int32),
                ("warm_inverse", C.c_int32), ("frag_block", C.c_int32), ("lu_param", C.c_int32)]


class GatedScanDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "length", "channels", "dtype", "input_gate", "reserved")] + \
               [(n, C.c_int64) for n in ("v_batch", "v_time", "f_batch", "f_time", "y_batch", "y_time",
                                         "dv_batch", "dv_time", "df_batch", "df_time")]


class ResidualNormDesc(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int32), ("dtype", C.c_int32), ("eps", C.c_double),
                ("ld_x", C.c_int64), ("ld_b", C.c_int64), ("ld_z", C.c_int64)]


class EmbeddingDesc(C.Structure):
    _fields_ = [("tokens", C.c_int64), ("vocab", C.c_int32), ("dim", C.c_int32), ("dtype", C.c_int32),
                ("grad_dtype", C.c_int32), ("index_bytes", C.c_int32), ("reserved", C.c_int32),
                ("ld_table", C.c_int64), ("ld_out", C.c_int64), ("ld_dtable", C.c_int64), ("scale", C.c_double)]


class TokenLossDesc(C.Structure):
    _fields_ = [("rows", C.c_int64), ("vocab", C.c_int32), ("dim", C.c_int32), ("dtype", C.c_int32),
                ("grad_dtype", C.c_int32), ("index_bytes", C.c_int32), ("piece_rows", C.c_int32),
                ("ld_h", C.c_int64), ("ld_weight", C.c_int64), ("ld_dh", C.c_int64), ("ld_dweight", C.c_int64),
                ("scale", C.c_double)]


class OrthDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("rows", "cols", "count", "prec", "steps", "nesterov", "terms",
                                         "reserved")] + [("coef", C.c_double * 3)]


_lib = None


def lib() -> C.CDLL:
    """Load the CUDA library (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} not found: build it with `python -m paper_2402_14212_b200.build`")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
        L.mw_net_create.argtypes = [C.POINTER(LayerDesc), i32, i32, C.POINTER(NetOpts), C.POINTER(vp)]
        L.mw_net_destroy.argtypes = [vp]
        L.mw_net_destroy.restype = None
        L.mw_workspace_bytes.argtypes = [vp, C.POINTER(sz), C.POINTER(sz), C.POINTER(sz)]
        L.mw_input_cotangent.argtypes = [vp, C.POINTER(vp), vp, vp, vp, vp, vp, sz, vp]
        L.mw_forward_sweep.argtypes = [vp, C.POINTER(vp), vp, vp, C.POINTER(vp), vp, sz, vp]
        L.mw_forward_sweep_apply.argtypes = [vp, C.POINTER(vp), vp, vp, C.c_double, C.POINTER(vp), vp, sz, vp]
        L.mw_sweep_bucket_events.argtypes = [vp, i32, C.POINTER(vp), i32]
        L.mw_backprop_reference.argtypes = [vp, C.POINTER(vp), vp, vp, C.POINTER(vp), vp, vp, sz, vp]
        L.mw_export_masks.argtypes = [vp, vp, i32, vp, sz, C.POINTER(i32), C.POINTER(i32), vp]
        L.mw_last_device_status.argtypes = [vp, vp, vp, C.POINTER(C.c_uint32)]
        L.mw_status_string.argtypes = [i32]
        L.mw_status_string.restype = C.c_char_p
        L.mw_pack_sign_bits.argtypes = [vp, i32, i64, i32, vp, vp]
        L.mw_relu_fragment_compact.argtypes = [vp, vp, i64, i32, vp, vp, vp, vp, vp, sz, vp]
        L.mw_activation_vijp.argtypes = [vp, vp, i64, i32, i32, C.c_float, vp, vp, vp, vp, vp]
        L.mw_gemm_split_bf16.argtypes = [vp, i32, vp, i32, vp, i32, i32, i32, i32, vp, sz, vp]
        L.mw_conv2d_split_bf16.argtypes = [i32, vp, vp, vp, i32, i32, i32, i32, i32, vp, sz, vp]
        L.mw_conv2d_strided_split_bf16.argtypes = [i32, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32,
                                                   i32, vp, sz, vp]
        L.mw_gemm_split_bf16_static.argtypes = [vp, i32, vp, i32, vp, i32, i32, i32, i32, vp]
        L.mw_gradient_step_host.argtypes = [vp, C.POINTER(vp), vp, sz, vp, sz, vp, vp, vp,
                                            C.POINTER(vp), vp, vp, vp, sz, vp]
        L.mw_launch_count.argtypes = []
        L.mw_launch_count.restype = C.c_int64
        L.mw_set_pair_mode.argtypes = [i32]
        L.mw_set_pair_mode.restype = i32
        L.mw_selftest_bounded_wait.argtypes = [vp, sz, C.c_uint32, C.POINTER(i32), vp]
        L.mw_set_sweep_chains.argtypes = [i32]
        L.mw_set_sweep_chains.restype = i32
        L.mw_set_bulk_epilogue.argtypes = [i32]
        L.mw_set_bulk_epilogue.restype = i32
        L.mw_set_cooperative_launch.argtypes = [i32]
        L.mw_set_cooperative_launch.restype = i32
        L.mw_set_merge_orders.argtypes = [i32]
        L.mw_set_merge_orders.restype = i32
        scan, norm, orth = C.POINTER(GatedScanDesc), C.POINTER(ResidualNormDesc), C.POINTER(OrthDesc)
        L.mw_gated_scan_states_bytes.argtypes = [scan, C.POINTER(sz)]
        L.mw_gated_scan_forward.argtypes = [scan] + [vp] * 9
        L.mw_gated_scan_backward.argtypes = [scan] + [vp] * 11
        L.mw_residual_norm_forward.argtypes = [norm] + [vp] * 10
        L.mw_residual_norm_scratch_bytes.argtypes = [norm, C.POINTER(sz)]
        L.mw_residual_norm_backward.argtypes = [norm] + [vp] * 16 + [sz, vp]
        L.mw_orth_create.argtypes = [orth, C.POINTER(vp)]
        L.mw_orth_destroy.argtypes = [vp]
        L.mw_orth_destroy.restype = None
        L.mw_orth_workspace_bytes.argtypes = [vp, C.POINTER(sz)]
        L.mw_orth_step.argtypes = [vp] + [C.POINTER(vp)] * 5 + [C.c_double] * 4 + [vp, sz, vp]
        L.mw_orth_project.argtypes = [vp, C.POINTER(vp), C.POINTER(vp), vp, sz, vp]
        L.mw_orth_status.argtypes = [vp, vp, vp]
        L.mw_orth_selftest_unmet_wait.argtypes = [vp, C.c_uint32]
        embed, tloss = C.POINTER(EmbeddingDesc), C.POINTER(TokenLossDesc)
        L.mw_embedding_forward.argtypes = [embed] + [vp] * 4
        L.mw_embedding_scratch_bytes.argtypes = [embed, C.POINTER(sz)]
        L.mw_embedding_backward.argtypes = [embed, vp, vp, vp, i32, vp, sz, vp]
        L.mw_token_loss_workspace_bytes.argtypes = [tloss, i32, C.POINTER(sz)]
        L.mw_token_loss_forward.argtypes = [tloss] + [vp] * 7 + [sz, vp]
        L.mw_token_loss_gradient.argtypes = [tloss] + [vp] * 9 + [sz, vp]
        L.mw_token_loss_status.argtypes = [vp, vp]
        L.mw_token_loss_selftest_unmet_wait.argtypes = [C.c_uint32, i32]
        L.mw_clip_scratch_bytes.argtypes = [i32, C.POINTER(sz)]
        L.mw_clip_gradients.argtypes = [i32, vp, vp, vp, vp, C.c_double, vp, vp, sz, vp]     # (arrays by their addresses)
        L.mw_profile_begin.argtypes = []
        L.mw_profile_begin.restype = None
        L.mw_profile_end.argtypes = [C.POINTER(C.c_double), C.POINTER(C.c_int64),
                                     C.POINTER(C.c_double), C.POINTER(C.c_double)]
        _lib = L
    return _lib


def _check(code: int, where: str):
    if code != MW_OK:
        raise MwError(code, where)


def _ptr(t) -> int:
    return 0 if t is None else int(t.data_ptr())


def _stream_handle(stream=None) -> int:
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return int(s.cuda_stream)


def _ptr_array(tensors: Sequence) -> "C.Array":
    arr = (C.c_void_p * len(tensors))()
    for i, t in enumerate(tensors):
        arr[i] = _ptr(t)
    return arr


def make_layer_descs(layers) -> "C.Array":
    arr = (LayerDesc * len(layers))()
    for i, l in enumerate(layers):
        arr[i] = LayerDesc(KIND[l.kind], ACT[l.act], float(l.slope), int(l.n_in), int(l.n_out),
                           int(l.H), int(l.W), int(l.C_in), int(l.C_out), int(l.k),
                           int(l.stride), int(l.pad))
    return arr


class Net:
    """Host-side handle of one network (mw_net).  Owns no device memory."""

    def __init__(self, layers, batch: int, prec: str, loss: str, reseed_every: int = 4,
                 conv_vijp_iters: int = 10, backend: str = "auto", inverse_iters: int = 0,
                 resident_inverse: bool = True, frag_block: int = 0, warm_inverse: bool = False):
        self.layers = list(layers)
        # LU-parameterised dense layers (Layer.lu): all layers of a net or none
        lu = [bool(getattr(l, "lu", False)) for l in self.layers]
        if any(lu) and not all(lu):
            raise ValueError("a net is LU-parameterised in every layer or in none")
        self.batch = int(batch)
        self.prec, self.loss = prec, loss
        self._h = C.c_void_p()
        opts = NetOpts(PREC[prec], LOSS[loss], int(reseed_every), int(conv_vijp_iters),
                       BACKEND[backend], int(inverse_iters), int(bool(resident_inverse)),
                       int(bool(warm_inverse)), int(frag_block), int(any(lu)))
        descs = make_layer_descs(self.layers)
        _check(lib().mw_net_create(descs, len(self.layers), self.batch, C.byref(opts),
                                   C.byref(self._h)), "mw_net_create")

    def close(self):
        if self._h:
            lib().mw_net_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- sizes -------------------------------------------------------------------------
    def workspace_bytes(self):
        a, b = C.c_size_t(), C.c_size_t()
        res = (C.c_size_t * 2)()
        _check(lib().mw_workspace_bytes(self._h, C.byref(a), C.byref(b), res), "mw_workspace_bytes")
        return int(a.value), int(b.value), (int(res[0]), int(res[1]))

    def grad_dtype(self):
        import torch
        return torch.float64 if self.prec == "f64" else torch.float32

    def storage_dtype(self):
        import torch
        return {"f64": torch.float64, "f32": torch.float32, "bf16_f32acc": torch.bfloat16}[self.prec]

    def alloc_workspace(self, which: str = "moonwalk", device="cuda"):
        import torch
        a, b, _ = self.workspace_bytes()
        n = a if which == "moonwalk" else (b if which == "backprop" else max(a, b))
        return torch.empty(n + 256, dtype=torch.uint8, device=device)

    @staticmethod
    def _ws(workspace):
        p = int(workspace.data_ptr())
        ap = (p + 255) // 256 * 256
        return ap, workspace.numel() - (ap - p)

    # ---- the three calls ------------------------------------------------------------------
    def input_cotangent(self, params, x, target, workspace, g0_out=None, loss_out=None, stream=None,
                        keep_seed=False):
        """keep_seed (nets of strided submersive convolutions only): g0 is not returned; the part
        of it that the sweep reads stays in the workspace (call forward_sweep with g0 = None)."""
        import torch
        if g0_out is None and not keep_seed:
            g0_out = torch.empty(x.shape, dtype=self.grad_dtype(), device=x.device)
        wp, wb = self._ws(workspace)
        _check(lib().mw_input_cotangent(self._h, _ptr_array(params), _ptr(x), _ptr(target),
                                        _ptr(g0_out), _ptr(loss_out), wp, wb,
                                        _stream_handle(stream)), "mw_input_cotangent")
        return g0_out

    def forward_sweep(self, params, x, g0, workspace, dW_out=None, stream=None):
        import torch
        if dW_out is None:
            dW_out = [torch.empty(p.shape, dtype=self.grad_dtype(), device=p.device) for p in params]
        wp, wb = self._ws(workspace)
        _check(lib().mw_forward_sweep(self._h, _ptr_array(params), _ptr(x), _ptr(g0),
                                      _ptr_array(dW_out), wp, wb, _stream_handle(stream)),
               "mw_forward_sweep")
        return dW_out

    def forward_sweep_apply(self, params, x, g0, lr: float, workspace, params_out=None, stream=None):
        """theta_l <- theta_l - lr * g_l inside the sweep; in place unless `params_out` is given."""
        if params_out is None:
            params_out = params
        wp, wb = self._ws(workspace)
        _check(lib().mw_forward_sweep_apply(self._h, _ptr_array(params), _ptr(x), _ptr(g0), float(lr),
                                            _ptr_array(params_out), wp, wb, _stream_handle(stream)),
               "mw_forward_sweep_apply")
        return params_out

    def set_bucket_events(self, layers_per_bucket: int, events=None):
        """events: torch.cuda.Event objects (already recorded once, so that their handles exist), one
        per bucket of `layers_per_bucket` layers; the forward sweep records them as the buckets'
        gradients are enqueued.  layers_per_bucket = 0 turns the feature off."""
        events = list(events or [])
        arr = (C.c_void_p * max(1, len(events)))()
        for i, e in enumerate(events):
            arr[i] = int(e.cuda_event)
        _check(lib().mw_sweep_bucket_events(self._h, int(layers_per_bucket), arr, len(events)),
               "mw_sweep_bucket_events")
        self._bucket_events = events          # keep them alive

    def backprop_reference(self, params, x, target, workspace, dW_out=None, loss_out=None,
                           stream=None):
        import torch
        if dW_out is None:
            dW_out = [torch.empty(p.shape, dtype=self.grad_dtype(), device=p.device) for p in params]
        wp, wb = self._ws(workspace)
        _check(lib().mw_backprop_reference(self._h, _ptr_array(params), _ptr(x), _ptr(target),
                                           _ptr_array(dW_out), _ptr(loss_out), wp, wb,
                                           _stream_handle(stream)), "mw_backprop_reference")
        return dW_out

    def gradient_step_host(self, params, x_host, target_host, x_dev, target_dev, g0_dev, dW_out,
                           loss_dev, loss_host, workspace, stream=None):
        """Whole step with the per-step inputs in (pinned) host memory; returns after the loss
        has landed in `loss_host`."""
        wp, wb = self._ws(workspace)
        _check(lib().mw_gradient_step_host(
            self._h, _ptr_array(params), _ptr(x_host), x_host.numel() * x_host.element_size(),
            _ptr(target_host), target_host.numel() * target_host.element_size(), _ptr(x_dev),
            _ptr(target_dev), _ptr(g0_dev), _ptr_array(dW_out), _ptr(loss_dev), _ptr(loss_host),
            wp, wb, _stream_handle(stream)), "mw_gradient_step_host")

    def export_masks(self, workspace, layer: int, stream=None) -> np.ndarray:
        l = self.layers[layer]
        if l.kind in ("conv2d", "conv1d"):
            ho, wo = l.out_hw()
            rows, cols = self.batch * ho * wo, l.C_out
        else:
            rows, cols = self.batch, l.n_out
        wpr = (cols + 31) // 32
        out = np.zeros((rows, wpr), dtype=np.uint32)
        wp, _ = self._ws(workspace)
        r, w = C.c_int32(), C.c_int32()
        _check(lib().mw_export_masks(self._h, wp, layer, out.ctypes.data, out.size, C.byref(r),
                                     C.byref(w), _stream_handle(stream)), "mw_export_masks")
        assert (r.value, w.value) == (rows, wpr)
        return out

    def last_device_status(self, workspace, stream=None):
        wp, _ = self._ws(workspace)
        detail = (C.c_uint32 * 4)()
        code = lib().mw_last_device_status(self._h, wp, _stream_handle(stream), detail)
        return code, list(detail)


def launch_count() -> int:
    return int(lib().mw_launch_count())


def set_pair_mode(enable: bool) -> bool:
    """Turn the CTA-pair form of the product kernel on or off; returns the previous setting."""
    return bool(lib().mw_set_pair_mode(int(bool(enable))))


def selftest_bounded_wait(limit_ms: int = 5, stream=None) -> int:
    """Run the library's self-test of its bounded device-side waits; returns the status that the
    deliberately unsatisfiable launch recorded (MW_ERR_TIMEOUT = 6 when the path works)."""
    import torch
    scratch = torch.empty(512 * 1024, dtype=torch.uint8, device="cuda")
    p = (int(scratch.data_ptr()) + 255) // 256 * 256
    out = C.c_int32(-1)
    _check(lib().mw_selftest_bounded_wait(p, scratch.numel() - 256, int(limit_ms), C.byref(out),
                                          _stream_handle(stream)), "mw_selftest_bounded_wait")
    return int(out.value)


def set_sweep_chains(mode: int) -> int:
    """Forward sweep of dense nets as per-row-block chains in one launch (1: form chosen by tile
    count, 2: CTA pairs whenever possible) or as a launch per layer (0).  Returns the old mode."""
    return int(lib().mw_set_sweep_chains(int(mode)))


def set_bulk_epilogue(enable: bool) -> bool:
    """Epilogue outputs through the copy engine (True) or per-lane stores (False)."""
    return bool(lib().mw_set_bulk_epilogue(int(bool(enable))))


def set_cooperative_launch(enable: bool) -> bool:
    """Program launches with or without the cooperative-launch attribute (profiling aid)."""
    return bool(lib().mw_set_cooperative_launch(int(bool(enable))))


def set_merge_orders(enable: bool) -> bool:
    """Two-term products of the pair form: one accumulator block for all cross products (True) or
    one per order (False); returns the previous setting."""
    return bool(lib().mw_set_merge_orders(int(bool(enable))))


def profile_begin():
    lib().mw_profile_begin()


def profile_end():
    ms, n, fl, mfl = C.c_double(), C.c_int64(), C.c_double(), C.c_double()
    _check(lib().mw_profile_end(C.byref(ms), C.byref(n), C.byref(fl), C.byref(mfl)), "mw_profile_end")
    return dict(total_ms=ms.value, launches=int(n.value), flops=fl.value, mma_flops=mfl.value)


# ---- stand-alone kernels -----------------------------------------------------------------
def pack_sign_bits(z, words=None, stream=None):
    import torch
    dt = {torch.float64: 0, torch.float32: 1, torch.bfloat16: 2}[z.dtype]
    rows, cols = z.shape
    if words is None:
        words = torch.zeros((rows, (cols + 31) // 32), dtype=torch.int32, device=z.device)
    _check(lib().mw_pack_sign_bits(_ptr(z), dt, rows, cols, _ptr(words), _stream_handle(stream)),
           "mw_pack_sign_bits")
    return words


def relu_fragment_compact(h, words, stream=None):
    import torch
    rows, cols = h.shape
    dev = h.device
    cnt = torch.zeros(max(rows, 1), dtype=torch.int32, device=dev)
    off = torch.zeros(max(rows, 1), dtype=torch.int32, device=dev)
    vals = torch.zeros(max(rows * cols, 1), dtype=torch.float32, device=dev)
    total = torch.zeros(1, dtype=torch.int32, device=dev)
    scratch = torch.empty(4 * (rows + 1024), dtype=torch.uint8, device=dev)
    _check(lib().mw_relu_fragment_compact(_ptr(h), _ptr(words), rows, cols, _ptr(cnt), _ptr(off),
                                          _ptr(vals), _ptr(total), _ptr(scratch), scratch.numel(),
                                          _stream_handle(stream)), "mw_relu_fragment_compact")
    return cnt[:rows], off[:rows], vals, total


def activation_vijp(gz, words, act: str, slope: float = 0.0, off=None, vals=None, want_gz=False,
                    stream=None):
    import torch
    rows, cols = gz.shape
    h = torch.empty_like(gz)
    gzo = torch.empty_like(gz) if want_gz else None
    _check(lib().mw_activation_vijp(_ptr(gz), _ptr(words), rows, cols, ACT[act], float(slope),
                                    _ptr(off), _ptr(vals), _ptr(h), _ptr(gzo),
                                    _stream_handle(stream)), "mw_activation_vijp")
    return (h, gzo) if want_gz else h


def gemm_split_bf16(A, B, a_mn: bool, b_mn: bool, terms: int, stream=None):
    """D = op(A) op(B)^T-style product on the tensor cores (see moonwalk.h)."""
    import torch
    M = A.shape[1] if a_mn else A.shape[0]
    K = A.shape[0] if a_mn else A.shape[1]
    N = B.shape[1] if b_mn else B.shape[0]
    D = torch.empty((M, N), dtype=torch.float32, device=A.device)
    scratch = torch.empty(6 * (M * K + N * K) + 4096, dtype=torch.uint8, device=A.device)
    _check(lib().mw_gemm_split_bf16(_ptr(A), int(a_mn), _ptr(B), int(b_mn), _ptr(D), M, N, K,
                                    int(terms), _ptr(scratch), scratch.numel(),
                                    _stream_handle(stream)), "mw_gemm_split_bf16")
    return D


def conv2d_split_bf16(op: int, a, b, k: int, terms: int, stream=None):
    """op 0: conv(a = x, b = w); op 1: TransposeConv(a = h', b = w); op 2: weight vjp (a = x, b = g_z)."""
    import torch
    images, H, W, C = a.shape
    assert C == 64
    out = torch.empty((k, k, 64, 64) if op == 2 else (images, H, W, 64), dtype=torch.float32,
                      device=a.device)
    n = 1024 + 8 * terms * (a.numel() + b.numel()) + 256 * k * k * 16384 + 4096
    scratch = torch.empty(n, dtype=torch.uint8, device=a.device)
    _check(lib().mw_conv2d_split_bf16(op, _ptr(a), _ptr(b), _ptr(out), images, H, W, k, int(terms),
                                      _ptr(scratch), scratch.numel(), _stream_handle(stream)),
           "mw_conv2d_split_bf16")
    return out


def conv2d_strided_split_bf16(op: int, a, b, k: int, stride: int, pad: int, terms: int, in_hw=None,
                              stream=None):
    """op 0: conv(a = x, b = w); op 1: TransposeConv(a = h', b = w) back to the `in_hw` image;
    op 2: weight vjp (a = x, b = g_z).  Channel-last float tensors, C channels in and out."""
    import torch
    images, Ha, Wa, C = a.shape
    if op == 1:
        H, W = in_hw
    else:
        H, W = Ha, Wa
    Ho, Wo = (H + 2 * pad - k) // stride + 1, (W + 2 * pad - k) // stride + 1
    shape = {0: (images, Ho, Wo, C), 1: (images, H, W, C), 2: (k, k, C, C)}[op]
    out = torch.empty(shape, dtype=torch.float32, device=a.device)
    n = 1024 + 8 * terms * (a.numel() + b.numel()) + 1024 * k * k * C * C + 4096
    scratch = torch.empty(n, dtype=torch.uint8, device=a.device)
    _check(lib().mw_conv2d_strided_split_bf16(op, _ptr(a), _ptr(b), _ptr(out), images, H, W, C, k,
                                              stride, pad, int(terms), _ptr(scratch), scratch.numel(),
                                              _stream_handle(stream)),
           "mw_conv2d_strided_split_bf16")
    return out


GEMM_STATIC_SCRATCH_BYTES = 16 << 20


def gemm_split_bf16_static(A, B, a_mn: bool, b_mn: bool, terms: int, stream=None):
    """mw_gemm_split_bf16_static: the same product with the library's built-in scratch, for callers
    that cannot allocate a scratch buffer.  Only the output tensor is created here (by torch, as
    for every other call of this binding); the C entry point itself allocates nothing."""
    import torch
    M = A.shape[1] if a_mn else A.shape[0]
    K = A.shape[0] if a_mn else A.shape[1]
    N = B.shape[1] if b_mn else B.shape[0]
    D = torch.empty((M, N), dtype=torch.float32, device=A.device)
    _check(lib().mw_gemm_split_bf16_static(_ptr(A), int(a_mn), _ptr(B), int(b_mn), _ptr(D), M, N, K,
                                           int(terms), _stream_handle(stream)),
           "mw_gemm_split_bf16_static")
    return D


# ---- layers in front of a net, and the optimiser's step --------------------------------------
INPUT_GATE = {"complement": 0, "energy": 1}
SCAN_STATE_EVERY = 16


def _operand_dtype(t, where: str) -> int:
    import torch
    codes = {torch.float32: 1, torch.bfloat16: 2}
    if t.dtype not in codes:
        raise TypeError(f"{where}: float32 or bfloat16 tensors, got {t.dtype}")
    return codes[t.dtype]


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _same_device(ref, named, where: str):
    for name, t in named.items():
        if t is not None:
            _need(t.device == ref.device, f"{where}: {name} is on {t.device}, not on {ref.device}")


def _check_float(t, shape, name, device):
    """Optional float32 contiguous tensor of a given shape."""
    import torch
    if t is not None:
        _need(t.dtype == torch.float32 and tuple(t.shape) == tuple(shape) and t.is_contiguous() and
              t.device == device, f"{name}: a contiguous float32 tensor of shape {tuple(shape)} on {device}")


# Descriptions of calls whose tensors have passed the checks below, by everything the checks look at (types,
# shapes, strides, devices): a serving loop pays for them once.
_passed = {}


def _layout(t):
    return None if t is None else (t.dtype, t.shape, t.stride(), t.device)


def _remember(key, value):
    if len(_passed) >= 4096:
        _passed.clear()
    _passed[key] = value
    return value


def _raw_stream(stream, device) -> int:
    """Handle of `stream`, or of the device's current stream."""
    import torch
    if stream is not None:
        return int(stream.cuda_stream)
    return torch._C._cuda_getCurrentRawStream(device.index)


def _current_device() -> int:
    import torch
    return torch._C._cuda_getDevice()


def _call(name, device, *args, stream=None) -> int:
    """A library call with `device` current, on `stream` or the device's current stream: the library launches, and
    asks for the number of SMs, on the current device.  Returns its status."""
    if stream is not None:
        _need(stream.device == device, f"{name}: a stream of {device}")
    call, handle = getattr(lib(), name), _raw_stream(stream, device)
    if _current_device() == device.index:
        return call(*args, handle)
    import torch
    with torch.cuda.device(device):
        return call(*args, handle)


def _keep_for(stream, *things):
    """Marks tensors (and lists of them) as used on `stream`: their memory is not given out again, should the caller
    drop them, before the work there is done."""
    import torch
    for t in things:
        if isinstance(t, torch.Tensor):
            t.record_stream(stream)
        elif isinstance(t, (list, tuple)):
            _keep_for(stream, *t)


def _on_stream(stream, like, call, *args):
    """call(*args) on `stream`.  What it allocates comes from that stream's memory, whose earlier uses lie
    before the call there, and what it hands back is kept until the caller's stream is done with it too; what it is
    given is kept until `stream` is.  `stream` does not wait for the caller's stream: that is the caller's to order."""
    import torch
    _need(stream.device == like.device, f"{call.__name__}: a stream of {like.device}, not of {stream.device}")
    with torch.cuda.stream(stream):
        out = call(*args)
    _keep_for(stream, *args)
    _keep_for(torch.cuda.current_stream(like.device), out)
    return out


def _dense_like(t):
    """A new dense tensor of t's shape and type."""
    import torch
    return torch.empty_like(t) if t.is_contiguous() else torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _repeats(t) -> bool:
    """Whether elements of t share memory by a stride of zero, as expanded tensors' do."""
    return t is not None and any(s == 0 and n > 1 for s, n in zip(t.stride(), t.shape))


def _own_memory(*tensors):
    """Each tensor, or a dense copy where it repeats elements: the library wants rows apart, and reads a stride of
    zero as the dense one."""
    return tuple(t.contiguous() if _repeats(t) else t for t in tensors)


def _scan_call(v, f, reset, lengths, input_gate, named):
    """Checks of the tensors every scan call shares; `named` {name: [B, T, D] tensor like v or None}."""
    import torch
    _need(v.is_cuda, "gated_scan: CUDA tensors")
    _need(v.dim() == 3, "gated_scan: v is [batch, length, channels]")
    if input_gate not in INPUT_GATE:
        raise ValueError(f"gated_scan: input_gate is one of {sorted(INPUT_GATE)}")
    B, T, D = v.shape
    d = GatedScanDesc(B, T, D, _operand_dtype(v, "gated_scan"), INPUT_GATE[input_gate], 0)
    # (a tensor without elements, or of one step or sequence, has strides that mean nothing)
    for name, field, t in [("v", "v", v), ("f", "f", f)] + named:
        if t is None:
            continue
        _need(t.dtype == v.dtype and tuple(t.shape) == (B, T, D), f"gated_scan: {name} has the type and shape of v")
        _need(D <= 1 or t.stride(2) == 1 or t.numel() == 0, f"gated_scan: {name}'s channels are contiguous")
        _need(not _repeats(t), f"gated_scan: {name} is written, and repeats elements")      # (inputs are copied before)
        if t.numel():
            setattr(d, field + "_batch", t.stride(0) if B > 1 else T * D)
            setattr(d, field + "_time", t.stride(1) if T > 1 else D)
    if reset is not None:
        _need(reset.dtype in (torch.uint8, torch.bool) and tuple(reset.shape) == (B, T) and reset.is_contiguous(),
              "gated_scan: reset is a contiguous uint8 or bool [batch, length]")
    if lengths is not None:
        _need(lengths.dtype == torch.int32 and tuple(lengths.shape) == (B,) and lengths.is_contiguous(),
              "gated_scan: lengths is a contiguous int32 [batch]")
    _same_device(v, dict({n: t for n, _, t in named}, f=f, reset=reset, lengths=lengths), "gated_scan")
    return d


def gated_scan(v, f, reset=None, lengths=None, h0=None, input_gate: str = "complement", keep_states=False,
               y=None, h_last=None, stream=None):
    """Gated linear recurrence h_t = r_t sigmoid(f_t) h_{t-1} + u_t v_t over dim 1 of [batch, length,
    channels] tensors (float32 or bfloat16; rows may be windows of wider ones; expanded ones are copied first).
    Returns (y, h_last), with keep_states=True (y, h_last, states) for gated_scan_backward.  One step
    (length 1) with h0 = h_last = the cached state is the serving form.  With `stream` the work runs there, after
    what that stream was given before: it does not wait for the current one."""
    import torch
    if stream is not None:
        return _on_stream(stream, v, gated_scan, v, f, reset, lengths, h0, input_gate, keep_states, y, h_last)
    key = ("scan", input_gate, keep_states, _layout(v), _layout(f), _layout(y), _layout(reset), _layout(lengths),
           _layout(h0), _layout(h_last))
    d = _passed.get(key)
    fresh = d is None
    if fresh and (_repeats(v) or _repeats(f)):
        return gated_scan(*_own_memory(v, f), reset, lengths, h0, input_gate, keep_states, y, h_last)
    if y is None:
        y = _dense_like(v)
    if fresh:
        d = _scan_call(v, f, reset, lengths, input_gate, [("y", "y", y)])
    B, T, D = v.shape
    if fresh:
        _check_float(h0, (B, D), "gated_scan: h0", v.device)
        _check_float(h_last, (B, D), "gated_scan: h_last", v.device)
        _remember(key, d)
    if h_last is None:
        h_last = torch.empty_like(h0) if h0 is not None else torch.empty((B, D), dtype=torch.float32, device=v.device)
    states = None
    if keep_states:
        states = torch.empty((B, -(-T // SCAN_STATE_EVERY), D), dtype=torch.float32, device=v.device)
    _check(_call("mw_gated_scan_forward", v.device, d, v.data_ptr(), f.data_ptr(), _ptr(reset), _ptr(lengths), _ptr(h0),
                 y.data_ptr(), h_last.data_ptr(), _ptr(states)), "mw_gated_scan_forward")
    return (y, h_last, states) if keep_states else (y, h_last)


def gated_scan_backward(v, f, dy, states, reset=None, lengths=None, h0=None, dh_last=None,
                        input_gate: str = "complement", dv=None, df=None, stream=None):
    """(dv, df, dh0) of gated_scan from the cotangents of y and h_last (either may be None) and the
    states that the forward call kept (they include h0, which is accepted for symmetry).  Gradients of expanded
    inputs come element by element, as if the inputs had been dense.  `stream` as in gated_scan."""
    import torch
    if stream is not None:
        return _on_stream(stream, v, gated_scan_backward, v, f, dy, states, reset, lengths, h0, dh_last, input_gate, dv, df)
    key = ("scan backward", input_gate, _layout(v), _layout(f), _layout(dy), _layout(states), _layout(reset),
           _layout(lengths), _layout(dh_last), _layout(dv), _layout(df))
    d = _passed.get(key)
    fresh = d is None
    if fresh and (_repeats(v) or _repeats(f) or _repeats(dy)):
        return gated_scan_backward(*_own_memory(v, f, dy), states, reset, lengths, h0, dh_last, input_gate, dv, df)
    if dv is None:
        dv = _dense_like(v)
    if df is None:
        df = _dense_like(f)
    B, T, D = v.shape
    if fresh:
        d = _scan_call(v, f, reset, lengths, input_gate, [("dy", "y", dy), ("dv", "dv", dv), ("df", "df", df)])
        _check_float(dh_last, (B, D), "gated_scan_backward: dh_last", v.device)
        _need(states is not None, "gated_scan_backward: states come from gated_scan(..., keep_states=True)")
        _check_float(states, (B, -(-T // SCAN_STATE_EVERY), D), "gated_scan_backward: states", v.device)
        _remember(key, d)
    dh0 = torch.empty_like(dh_last) if dh_last is not None else torch.empty((B, D), dtype=torch.float32, device=v.device)
    _check(_call("mw_gated_scan_backward", v.device, d, v.data_ptr(), f.data_ptr(), _ptr(reset), _ptr(lengths),
                 states.data_ptr(), _ptr(dy), _ptr(dh_last), dv.data_ptr(), df.data_ptr(), dh0.data_ptr()),
           "mw_gated_scan_backward")
    return dv, df, dh0


def _norm_call(x, b, z, w_post, scale, w_pre, eps, dense):
    _need(x.is_cuda, "residual_norm: CUDA tensors")
    _need(x.dim() == 2, "residual_norm: x is [rows, cols]")
    R, D = x.shape
    d = ResidualNormDesc(R, D, _operand_dtype(x, "residual_norm"), float(eps), 0, 0, 0)
    for name, t in (("x", x), ("b", b), ("z", z)):
        if t is None:
            continue
        _need(t.dtype == x.dtype and tuple(t.shape) == (R, D), f"residual_norm: {name} has the type and shape of x")
        _need(D <= 1 or t.stride(1) == 1 or t.numel() == 0, f"residual_norm: {name}'s columns are contiguous")
        _need(not _repeats(t), f"residual_norm: {name} repeats elements")       # (copied before)
        setattr(d, "ld_" + name, t.stride(0) if R > 1 and t.numel() else D)
    for name, t in dense.items():
        if t is not None:
            _need(t.dtype == x.dtype and tuple(t.shape) == (R, D) and t.is_contiguous(),
                  f"residual_norm: {name} is contiguous, of x's type and shape")
    for name, t in (("w_post", w_post), ("scale", scale), ("w_pre", w_pre)):
        _check_float(t, (D,), "residual_norm: " + name, x.device)
    _same_device(x, dict(dense, b=b, z=z), "residual_norm")
    return d


def residual_norm(x, b=None, z=None, w_post=None, scale=None, w_pre=None, eps: float = 1e-6, keep_rms=False,
                  x_out=None, n=None, stream=None):
    """x' = x + scale silu(z) rmsnorm(b; w_post) and n = rmsnorm(x'; w_pre) on [rows, cols] tensors; what
    is None is left out (expanded x, b, z are copied first).  Returns (x', n), with keep_rms=True (x', n, inv_rms)
    for the backward call.  `stream` as in gated_scan."""
    import torch
    if stream is not None:
        return _on_stream(stream, x, residual_norm, x, b, z, w_post, scale, w_pre, eps, keep_rms, x_out, n)
    key = ("norm", eps, _layout(x), _layout(b), _layout(z), _layout(w_post), _layout(scale), _layout(w_pre),
           _layout(x_out), _layout(n))
    d = _passed.get(key)
    fresh = d is None
    if fresh and (_repeats(x) or _repeats(b) or _repeats(z)):
        x, b, z = _own_memory(x, b, z)
        return residual_norm(x, b, z, w_post, scale, w_pre, eps, keep_rms, x_out, n)
    if x_out is None:
        x_out = _dense_like(x)
    if n is None and w_pre is not None:
        n = _dense_like(x)
    if fresh:
        d = _remember(key, _norm_call(x, b, z, w_post, scale, w_pre, eps, {"x_out": x_out, "n": n}))
    rms = torch.empty((2, x.shape[0]), dtype=torch.float32, device=x.device) if keep_rms else None
    _check(_call("mw_residual_norm_forward", x.device, d, x.data_ptr(), _ptr(b), _ptr(z), _ptr(w_post), _ptr(scale),
                 _ptr(w_pre), x_out.data_ptr(), _ptr(n), _ptr(rms)), "mw_residual_norm_forward")
    return (x_out, n, rms) if keep_rms else (x_out, n)


class ResidualNormGrads(NamedTuple):
    dx: object
    db: object
    dz: object
    dw_post: object
    dscale: object
    dw_pre: object


def residual_norm_backward(x, b, inv_rms, z=None, w_post=None, scale=None, w_pre=None, eps: float = 1e-6,
                           dx_out=None, dn=None, stream=None) -> ResidualNormGrads:
    """Gradients of residual_norm from the cotangents of x' and n (either may be None); the gradients of
    what was left out are None, those of expanded inputs as if they had been dense.  `stream` as in gated_scan."""
    import torch
    if stream is not None:
        return _on_stream(stream, x, residual_norm_backward, x, b, inv_rms, z, w_post, scale, w_pre, eps, dx_out, dn)
    key = ("norm backward", eps, _layout(x), _layout(b), _layout(inv_rms), _layout(z), _layout(w_post),
           _layout(scale), _layout(w_pre), _layout(dx_out), _layout(dn))
    known = _passed.get(key)
    if known is None and (_repeats(x) or _repeats(b) or _repeats(z)):
        x, b, z = _own_memory(x, b, z)
        return residual_norm_backward(x, b, inv_rms, z, w_post, scale, w_pre, eps, dx_out, dn)
    if known is None:
        d = _norm_call(x, b, z, w_post, scale, w_pre, eps, {"dx_out": dx_out, "dn": dn})
        _need(inv_rms is not None, "residual_norm_backward: inv_rms comes from residual_norm(..., keep_rms=True)")
        _check_float(inv_rms, (2, x.shape[0]), "residual_norm_backward: inv_rms", x.device)
        need = C.c_size_t()
        with torch.cuda.device(x.device):          # (a partial sum a block, and blocks go by the device's SMs)
            _check(lib().mw_residual_norm_scratch_bytes(d, need), "mw_residual_norm_scratch_bytes")
        known = _remember(key, (d, int(need.value)))
    d, need = known
    g = ResidualNormGrads(*(None if t is None else _dense_like(t) for t in (x, b, z, w_post, scale, w_pre)))
    scratch = torch.empty(need, dtype=torch.uint8, device=x.device)
    _check(_call(
        "mw_residual_norm_backward", x.device, d, x.data_ptr(), _ptr(b), _ptr(z), _ptr(w_post), _ptr(scale), _ptr(w_pre),
        inv_rms.data_ptr(), _ptr(dx_out), _ptr(dn), g.dx.data_ptr(), _ptr(g.db), _ptr(g.dz), _ptr(g.dw_post),
        _ptr(g.dscale), _ptr(g.dw_pre), scratch.data_ptr(), need), "mw_residual_norm_backward")
    return g


class Orth:
    """Host-side handle of the orthogonalised update (mw_orth) of `count` weights of one shape.  Owns no
    device memory.  `prec` is the weights' storage; `terms` the accuracy of X: 1 (about 1e-3, the default for bf16
    weights that are neither small nor of few rows) or 2 (fp32 accuracy at three times the work, the default
    elsewhere)."""

    def __init__(self, rows: int, cols: int, count: int = 1, prec: str = "f32", steps: int = 0,
                 nesterov: bool = True, terms: int = 0, coef=(0.0, 0.0, 0.0)):
        self._h = C.c_void_p()
        self.shape, self.count, self.prec = (int(rows), int(cols)), int(count), prec
        d = OrthDesc(int(rows), int(cols), int(count), PREC[prec], int(steps), int(bool(nesterov)), int(terms), 0,
                     (C.c_double * 3)(*coef))
        _check(lib().mw_orth_create(C.byref(d), C.byref(self._h)), "mw_orth_create")

    def close(self):
        if self._h:
            lib().mw_orth_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def storage_dtype(self):
        import torch
        return {"f32": torch.float32, "bf16_f32acc": torch.bfloat16}[self.prec]

    def workspace_bytes(self) -> int:
        n = C.c_size_t()
        _check(lib().mw_orth_workspace_bytes(self._h, C.byref(n)), "mw_orth_workspace_bytes")
        return int(n.value)

    def alloc_workspace(self, device="cuda"):
        import torch
        return torch.empty(self.workspace_bytes() + 256, dtype=torch.uint8, device=device)

    def _list(self, tensors, dtype, name, workspace):
        tensors = list(tensors)
        ok = len(tensors) == self.count and workspace.is_cuda
        for t in tensors:
            ok = ok and t.dtype == dtype and t.shape == self.shape and t.is_contiguous() and t.device == workspace.device
        if not ok:
            raise ValueError(f"Orth: {name} are {self.count} contiguous {dtype} tensors of shape {self.shape} on the "
                             "workspace's CUDA device")
        return (C.c_void_p * self.count)(*[t.data_ptr() for t in tensors])

    def step(self, params, grads, momentum, workspace, lr: float, beta: float = 0.95, weight_decay: float = 0.0,
             scale: float = 1.0, params_out=None, momentum_out=None, stream=None):
        """M <- beta M + G, W <- (1 - lr weight_decay) W - lr scale X; in place unless outputs are given.  With
        `stream` the work runs there, after what that stream was given before.  Where status() then tells of a wait
        that ran out, the weights are as they were."""
        import torch
        params_out = params if params_out is None else params_out
        momentum_out = momentum if momentum_out is None else momentum_out
        st, f32 = self.storage_dtype(), torch.float32
        wp, wb = Net._ws(workspace)
        _check(_call(
            "mw_orth_step", workspace.device, self._h, self._list(params, st, "params", workspace),
            self._list(grads, f32, "grads", workspace),
            self._list(momentum, f32, "momentum", workspace), self._list(params_out, st, "params_out", workspace),
            self._list(momentum_out, f32, "momentum_out", workspace), float(lr), float(beta), float(weight_decay), float(scale),
            wp, wb, stream=stream), "mw_orth_step")
        if stream is not None:
            _keep_for(stream, params, grads, momentum, params_out, momentum_out, workspace)
        return params_out

    def project(self, mats, workspace, out=None, stream=None):
        """The orthogonalised factor X of every matrix, in the storage type; on `stream` as in step()."""
        import torch
        if stream is not None:
            return _on_stream(stream, workspace, self.project, list(mats), workspace, out)
        st = self.storage_dtype()
        if out is None:
            out = [torch.empty_like(t) for t in mats]
        wp, wb = Net._ws(workspace)
        _check(_call("mw_orth_project", workspace.device, self._h, self._list(mats, st, "mats", workspace),
                     self._list(out, st, "out", workspace), wp, wb), "mw_orth_project")
        return out

    def selftest_unmet_wait(self, limit_ms: int):
        """The next calls hold a wait that nothing meets and that runs out after limit_ms (0 ends it)."""
        _check(lib().mw_orth_selftest_unmet_wait(self._h, int(limit_ms)), "mw_orth_selftest_unmet_wait")

    def status(self, workspace, stream=None) -> int:
        """Waits for the stream; the first device-side error of the last call on this workspace (0: none)."""
        wp, _ = Net._ws(workspace)
        return int(_call("mw_orth_status", workspace.device, self._h, wp, stream=stream))


# ---- the two ends of a token model, and the bound of its step ----------------------------------
def _index_bytes(t, where: str) -> int:
    import torch
    if t.dtype not in (torch.int32, torch.int64):
        raise TypeError(f"{where}: int32 or int64, got {t.dtype}")
    return 4 if t.dtype == torch.int32 else 8


def _grad_code(dtype, own, where: str):
    """(torch type, code) of a weight gradient: `dtype`, or the weight's own type where None."""
    import torch
    dtype = own if dtype is None else dtype
    if dtype not in (torch.float32, torch.bfloat16):
        raise TypeError(f"{where}: a gradient in float32 or bfloat16, got {dtype}")
    return dtype, 1 if dtype == torch.float32 else 2


def _rows_apart(t, name):
    """Elements between the rows of a [rows, columns] tensor whose columns are contiguous."""
    _need(t.shape[1] <= 1 or t.stride(1) == 1 or t.numel() == 0, f"{name}: columns are contiguous")
    return t.stride(0) if t.shape[0] > 1 and t.numel() else max(1, t.shape[1])


def _table_rows(t, name):
    _need(t.dim() == 2 and t.shape[0] >= 1 and t.shape[1] >= 1, f"{name}: [vocabulary, columns], neither zero")
    return _rows_apart(t, name)


def embedding(tokens, table, scale: float = 1.0, out=None, stream=None):
    """out = scale * table[tokens]: tokens int32 or int64 of any shape, table [vocabulary, columns] float32 or
    bfloat16 (rows may be windows of wider ones), out [*tokens.shape, columns].  A token that is no row of the
    table gives zeros.  `stream` as in gated_scan."""
    import torch
    if stream is not None:
        return _on_stream(stream, table, embedding, tokens, table, scale, out)
    key = ("embedding", scale, _layout(tokens), _layout(table), _layout(out))
    d = _passed.get(key)
    fresh = d is None
    if fresh and (_repeats(table) or not tokens.is_contiguous()):
        return embedding(tokens.contiguous(), *_own_memory(table), scale, out)
    if fresh:
        _need(table.is_cuda, "embedding: CUDA tensors")
        d = EmbeddingDesc(tokens.numel(), table.shape[0], table.shape[-1], _operand_dtype(table, "embedding"), 0,
                          _index_bytes(tokens, "embedding: tokens"), 0, _table_rows(table, "embedding: table"), 0, 0, float(scale))
        if out is not None:
            _need(out.dtype == table.dtype and tuple(out.shape) == (*tokens.shape, table.shape[1]) and out.is_contiguous(),
                  "embedding: out is contiguous, of the table's type and shape [*tokens.shape, columns]")
        _same_device(table, dict(tokens=tokens, out=out), "embedding")
    if out is None:
        out = torch.empty((*tokens.shape, table.shape[1]), dtype=table.dtype, device=table.device)
    _check(_call("mw_embedding_forward", table.device, d, tokens.data_ptr(), table.data_ptr(), out.data_ptr()),
           "mw_embedding_forward")
    if fresh:
        _remember(key, d)
    return out


def embedding_backward(tokens, dout, vocab: int, scale: float = 1.0, dtable=None, accumulate: bool = False,
                       grad_dtype=None, stream=None):
    """Gradient [vocab, columns] of embedding's table from dout [*tokens.shape, columns], summed in float32 in the
    order of the tokens; grad_dtype: float32 or bfloat16 (dout's where None).  With accumulate the rows that tokens
    name are added to dtable, whose other rows stay as they are.  `stream` as in gated_scan."""
    import torch
    if stream is not None:
        return _on_stream(stream, dout, embedding_backward, tokens, dout, vocab, scale, dtable, accumulate, grad_dtype)
    key = ("embedding backward", vocab, scale, bool(accumulate), grad_dtype, _layout(tokens), _layout(dout), _layout(dtable))
    known = _passed.get(key)
    if known is None:
        _need(dout.is_cuda, "embedding_backward: CUDA tensors")
        _need(dout.dim() >= 1 and tuple(dout.shape[:-1]) == tuple(tokens.shape) and dout.shape[-1] >= 1,
              "embedding_backward: dout is [*tokens.shape, columns]")
        rows = dout if dout.dim() == 2 else None
        if _repeats(dout) or not tokens.is_contiguous() or (rows is None and not dout.is_contiguous()):
            return embedding_backward(tokens.contiguous(), dout.contiguous(), vocab, scale, dtable, accumulate, grad_dtype)
        _need(not accumulate or dtable is not None, "embedding_backward: accumulate adds to a dtable")
        kind, code = _grad_code(dtable.dtype if dtable is not None and grad_dtype is None else grad_dtype, dout.dtype,
                                "embedding_backward")
        d = EmbeddingDesc(tokens.numel(), int(vocab), dout.shape[-1], _operand_dtype(dout, "embedding_backward"), code,
                          _index_bytes(tokens, "embedding_backward: tokens"), 0, 0,
                          _rows_apart(rows, "embedding_backward: dout") if rows is not None else 0, 0, float(scale))
        if dtable is not None:
            _need(dtable.dtype == kind and tuple(dtable.shape) == (vocab, dout.shape[-1]) and not _repeats(dtable),
                  f"embedding_backward: dtable is [{vocab}, {dout.shape[-1]}] of {kind}")
            d.ld_dtable = _table_rows(dtable, "embedding_backward: dtable")
        _same_device(dout, dict(tokens=tokens, dtable=dtable), "embedding_backward")
        need = C.c_size_t()
        _check(lib().mw_embedding_scratch_bytes(d, need), "mw_embedding_scratch_bytes")
        known = (d, int(need.value), kind)
        _remember(key, known)
    d, need, kind = known
    if dtable is None:
        dtable = torch.empty((vocab, dout.shape[-1]), dtype=kind, device=dout.device)
    scratch = torch.empty(need, dtype=torch.uint8, device=dout.device)
    _check(_call("mw_embedding_backward", dout.device, d, tokens.data_ptr(), dout.data_ptr(), dtable.data_ptr(),
                 int(bool(accumulate)), scratch.data_ptr(), need), "mw_embedding_backward")
    return dtable


class TokenLoss(NamedTuple):
    loss: object          # float32 [rows]
    total: object         # float32 []
    dh: object = None
    dweight: object = None


def token_loss_workspace(h, weight, gradient: bool = False, piece_rows: int = 0):
    """Memory for token_loss (or token_loss_gradient) calls with this h and weight, for their `workspace`."""
    import torch
    _need(h.is_cuda and h.dim() == 2 and weight.dim() == 2, "token_loss_workspace: CUDA tensors [rows, columns]")
    d = TokenLossDesc(h.shape[0], weight.shape[0], h.shape[1], _operand_dtype(h, "token_loss_workspace"), 0, 8, int(piece_rows), 0, 0,
                      0, 0, 1.0)
    need, most = C.c_size_t(), 0
    rows_apart = weight.shape[1] if _repeats(weight) else _table_rows(weight, "token_loss_workspace: weight")
    with torch.cuda.device(h.device):
        for d.ld_weight in {rows_apart, weight.shape[1]}:          # (as it is, or copied)
            _check(lib().mw_token_loss_workspace_bytes(d, int(bool(gradient)), need), "mw_token_loss_workspace_bytes")
            most = max(most, int(need.value))
    return torch.empty(most + 256, dtype=torch.uint8, device=h.device)


def token_loss_status(workspace, stream=None) -> int:
    """Waits for the stream; the first device-side error of the last token_loss or token_loss_gradient call on this
    workspace (0: none)."""
    wp, _ = Net._ws(workspace)
    return int(_call("mw_token_loss_status", workspace.device, wp, stream=stream))


def token_loss_selftest_unmet_wait(limit_ms: int, product: int = 0):
    """The calls of this thread hold a wait that nothing meets and that runs out after limit_ms (0 ends it): in the
    product of the logits (0), of dh (1) or of dweight (2)."""
    _check(lib().mw_token_loss_selftest_unmet_wait(int(limit_ms), int(product)), "mw_token_loss_selftest_unmet_wait")


def _token_loss(gradient, h, weight, targets, scale, row_weight, piece_rows, grad_dtype, dh, dweight, want, workspace=None):
    import torch
    key = ("token loss", gradient, scale, piece_rows, grad_dtype, want, _layout(h), _layout(weight), _layout(targets),
           _layout(row_weight), _layout(dh), _layout(dweight))
    known = _passed.get(key)
    if known is None:
        _need(h.is_cuda, "token_loss: CUDA tensors")
        if _repeats(h) or _repeats(weight):
            h, weight = _own_memory(h, weight)
            return _token_loss(gradient, h, weight, targets, scale, row_weight, piece_rows, grad_dtype, dh, dweight, want, workspace)
        _need(h.dim() == 2 and weight.dim() == 2 and h.shape[1] == weight.shape[1] and h.dtype == weight.dtype,
              "token_loss: h is [rows, columns], weight [vocabulary, columns] of the same type")
        _need(tuple(targets.shape) == (h.shape[0],) and targets.is_contiguous(), "token_loss: targets are contiguous, [rows]")
        _check_float(row_weight, (h.shape[0],), "token_loss: row_weight", h.device)
        kind, code = _grad_code(dweight.dtype if dweight is not None and grad_dtype is None else grad_dtype, weight.dtype,
                                "token_loss")
        d = TokenLossDesc(h.shape[0], weight.shape[0], h.shape[1], _operand_dtype(h, "token_loss"), code,
                          _index_bytes(targets, "token_loss: targets"), int(piece_rows), 0,
                          _table_rows(weight, "token_loss: weight"), 0, 0, float(scale))
        d.ld_h = _rows_apart(h, "token_loss: h")
        if dh is not None:
            _need(dh.dtype == h.dtype and dh.shape == h.shape and not _repeats(dh), "token_loss: dh has the type and shape of h")
            d.ld_dh = _rows_apart(dh, "token_loss: dh")
        if dweight is not None:
            _need(dweight.dtype == kind and dweight.shape == weight.shape and not _repeats(dweight),
                  f"token_loss: dweight is {kind} of weight's shape")
            d.ld_dweight = _table_rows(dweight, "token_loss: dweight")
        _same_device(h, dict(weight=weight, targets=targets, dh=dh, dweight=dweight), "token_loss")
        need = C.c_size_t()
        with torch.cuda.device(h.device):          # (some of it goes by the device's multiprocessors)
            _check(lib().mw_token_loss_workspace_bytes(d, int(gradient), need), "mw_token_loss_workspace_bytes")
        known = _remember(key, (d, int(need.value), kind))
    d, need, kind = known
    device = h.device
    loss = torch.empty(h.shape[0], dtype=torch.float32, device=device)
    total = torch.empty((), dtype=torch.float32, device=device)
    if workspace is None:
        ws = torch.empty(need, dtype=torch.uint8, device=device)
        at = ws.data_ptr()
    else:
        _need(workspace.dtype == torch.uint8 and workspace.is_contiguous() and workspace.device == device,
              f"token_loss: workspace is of bytes (uint8) on {device}")
        at, room = Net._ws(workspace)
        _need(room >= need, f"token_loss: workspace of {need} bytes from a multiple of 256 on")
    if not gradient:
        _check(_call("mw_token_loss_forward", device, d, h.data_ptr(), weight.data_ptr(), targets.data_ptr(),
                     _ptr(row_weight), loss.data_ptr(), total.data_ptr(), at, need), "mw_token_loss_forward")
        return TokenLoss(loss, total)
    if dh is None and want[0]:
        dh = _dense_like(h)
    if dweight is None and want[1]:
        dweight = torch.empty(weight.shape, dtype=kind, device=device)
    _check(_call("mw_token_loss_gradient", device, d, h.data_ptr(), weight.data_ptr(), targets.data_ptr(),
                 _ptr(row_weight), loss.data_ptr(), total.data_ptr(), _ptr(dh), _ptr(dweight), at, need),
           "mw_token_loss_gradient")
    return TokenLoss(loss, total, dh, dweight)


def token_loss(h, weight, targets, scale: float = 1.0, row_weight=None, stream=None, workspace=None) -> TokenLoss:
    """Softmax cross entropy of z = scale * h weight^T over a vocabulary, the logits never held: h [rows, columns]
    and weight [vocabulary, columns] float32 or bfloat16, targets int32 or int64 [rows].  Rows whose target is no row
    of weight (a negative one, say), or whose row_weight is zero, are left out: their loss is zero and their h is
    not read into anything.  total = sum of row_weight * loss, the mean over the rows that are left without
    row_weight.  workspace: memory of token_loss_workspace, which no other call in flight uses and from which
    token_loss_status reads whether all went well; a call's own otherwise.  `stream` as in gated_scan."""
    import torch
    if stream is not None:
        return _on_stream(stream, h, token_loss, h, weight, targets, scale, row_weight, None, workspace)
    if weight.dtype == torch.bfloat16 and weight.data_ptr() & 15:         # (read in place, by copies of 16 bytes)
        weight = weight.clone(memory_format=torch.contiguous_format)
    return _token_loss(False, h, weight, targets, scale, row_weight, 0, None, None, None, (False, False), workspace)


def token_loss_gradient(h, weight, targets, scale: float = 1.0, row_weight=None, dh=None, dweight=None,
                        grad_dtype=None, want=(True, True), piece_rows: int = 0, stream=None, workspace=None) -> TokenLoss:
    """token_loss, and the gradients of its total: dh (zero in rows left out; may be h itself) and dweight
    (float32 or bfloat16 by grad_dtype, weight's type where None).  want: which of the two.  piece_rows: rows whose
    exponentials are held at a time (0: as many as take 1 GiB); fewer take less memory and more time.  dz of bf16
    operands has 11 bits, which a float32 dweight shows.  `workspace` as in token_loss, `stream` as in gated_scan."""
    import torch
    if stream is not None:
        return _on_stream(stream, h, token_loss_gradient, h, weight, targets, scale, row_weight, dh, dweight, grad_dtype,
                          want, piece_rows, None, workspace)
    # (of few rows read in place, by copies of 16 bytes)
    if weight.dtype == torch.bfloat16 and weight.data_ptr() & 15 and targets.numel() <= 128:
        weight = weight.clone(memory_format=torch.contiguous_format)
    return _token_loss(True, h, weight, targets, scale, row_weight, piece_rows, grad_dtype, dh, dweight,
                       (bool(want[0]), bool(want[1])), workspace)


def clip_gradients(grads, max_norm: float, out=None, stream=None):
    """Scales the tensors together so that their common norm is at most max_norm; in place unless `out` gives a
    tensor for each.  Contiguous float32 or bfloat16 tensors of any shapes on one device, none of which shares memory
    with another (a weight used twice has one gradient).  Returns the norm before, a float32 tensor of no dimensions;
    where it is not finite the gradients stay as they are, and a step that looks at it leaves its weights alone.
    max_norm infinite: the norm alone.  `stream` as in gated_scan."""
    import torch
    grads = list(grads)
    _need(len(grads) > 0, "clip_gradients: at least one tensor")
    out = grads if out is None else list(out)
    if stream is not None:
        return _on_stream(stream, grads[0], clip_gradients, grads, max_norm, out)
    n, device, place = len(grads), grads[0].device, {grads[0].get_device()}
    _need(grads[0].is_cuda and len(out) == n, "clip_gradients: CUDA tensors, and as many outputs")
    Tensor, in_place = torch.Tensor, all(map(operator.is_, grads, out))
    # (whole lists at a time: a step has hundreds of tensors, and the loop over them is the call's time)
    kinds, sizes = [g.dtype for g in grads], list(map(Tensor.numel, grads))
    ok = all(map(Tensor.is_contiguous, grads)) and set(map(Tensor.get_device, grads)) == place
    if not in_place:
        ok = ok and all(map(Tensor.is_contiguous, out)) and set(map(Tensor.get_device, out)) == place
        ok = ok and kinds == [o.dtype for o in out] and sizes == list(map(Tensor.numel, out))
    codes = {torch.float32: 1, torch.bfloat16: 2}
    if not ok or not codes.keys() >= set(kinds):
        raise ValueError("clip_gradients: contiguous float32 or bfloat16 tensors on one device, outputs like them")
    need = _passed.get(("clip", n))
    if need is None:
        size = C.c_size_t()
        _check(lib().mw_clip_scratch_bytes(n, size), "mw_clip_scratch_bytes")
        need = _remember(("clip", n), int(size.value))
    norm = torch.empty((), dtype=torch.float32, device=device)
    scratch = torch.empty(need, dtype=torch.uint8, device=device)
    src = array.array("Q", map(Tensor.data_ptr, grads))
    dst = src if in_place else array.array("Q", map(Tensor.data_ptr, out))
    sizes, kinds = array.array("q", sizes), array.array("i", map(codes.__getitem__, kinds))
    at = [a.buffer_info()[0] for a in (src, dst, sizes, kinds)]
    _check(_call("mw_clip_gradients", device, n, *at, float(max_norm), norm.data_ptr(), scratch.data_ptr(), need),
           "mw_clip_gradients")
    return norm


# ---- moving a synthetic problem onto the device -------------------------------------------
def to_device(problem, device="cuda"):
    """Returns (params, x, target) as torch tensors in the problem's storage types."""
    import torch
    st = {"f64": torch.float64, "f32": torch.float32, "bf16_f32acc": torch.bfloat16}[problem.prec]
    gt = torch.float64 if problem.prec == "f64" else torch.float32
    params = [torch.from_numpy(np.ascontiguousarray(p)).to(st).to(device).contiguous()
              for p in problem.params]
    x = torch.from_numpy(np.ascontiguousarray(problem.x)).to(st).to(device).contiguous()
    if problem.loss == "xent_mean":
        target = torch.from_numpy(problem.target.astype(np.int32)).to(device)
    else:
        target = torch.from_numpy(np.ascontiguousarray(problem.target)).to(gt).to(device).contiguous()
    return params, x, target


def net_for(problem, backend="auto", resident_inverse=True, inverse_iters=0, warm_inverse=False) -> Net:
    return Net(problem.layers, problem.batch, problem.prec, problem.loss,
               reseed_every=problem.reseed_every, conv_vijp_iters=problem.conv_vijp_iters,
               backend=backend, inverse_iters=inverse_iters, resident_inverse=resident_inverse,
               frag_block=getattr(problem, "frag_block", 0), warm_inverse=warm_inverse)
