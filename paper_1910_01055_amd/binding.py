"""Thin ctypes binding over libactorq.so (the C ABI in include/actorq.h).

Argument marshalling only: every step of the path runs in the library's HIP kernels.
PyTorch supplies device memory (tensors) and the current HIP stream, nothing else.
There is no fallback: if the library is not built, load() raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libactorq.so")
MAX_LAYERS = 8

OK, EINVAL, ESHAPE, ENONFINITE, ENOTQUANT, EHIP, ENOMEM, ERANGE, ETOOBIG = range(9)
STATIC_SCRATCH_BYTES = 16 << 20
KIND = {"fc": 0, "conv": 1}
ACT = {"none": 0, "relu": 1, "ln_tanh": 2}
HEAD = {"tanh": 0, "argmax": 1, "linear": 2}
WSCHEME = {"tensor_asym_u8": 0, "channel_sym_s8": 1}
INTYPE = {"f32": 0, "u8": 1}

EXPORTS = ["aq_policy_create", "aq_policy_destroy", "aq_policy_reserve", "aq_policy_set_path", "aq_policy_status",
           "aq_quantize_tensor", "aq_quantize_params", "aq_policy_export_layer", "aq_policy_export_act_qparams",
           "aq_policy_forward_int8", "aq_policy_forward_fp32", "aq_status_string",
           "aq_policy_blob_size", "aq_policy_export_blob", "aq_policy_import_blob", "aq_policy_explore", "aq_policy_step_int8",
           "aq_convert_params_fp16", "aq_policy_forward_fp16",
           "aq_policy_packed_blob_size", "aq_policy_export_packed_blob", "aq_policy_import_packed_blob",
           "aq_policy_conv_stack_layers", "aq_policy_fp16_conv_stack_layers", "aq_policy_fused_plan", "aq_policy_forward_int8_static",
           "aq_policy_set_params_fp32", "aq_calibrate_fp32", "aq_policy_forward_fp32_params", "aq_stream_reference",
           "aq_mfma_loop_reference", "aq_policy_subbyte_layers", "aq_policy_fp32_plan", "aq_policy_fp16_plan",
           "aq_layernorm_forward", "aq_layernorm_backward", "aq_layernorm_backward_workspace", "aq_ckpt8_pack", "aq_ckpt8_unpack",
           "aq_ckpt8_weight_grad", "aq_ckpt8_weight_grad_workspace", "aq_mx4_quantize", "aq_mx4_dequantize", "aq_mx4_linear",
           "aq_mx4_linear_workspace", "aq_mx4_matmul", "aq_mx4_input_grad", "aq_mx4_input_grad_workspace"]


class AqLayer(C.Structure):
    _fields_ = [("kind", C.c_int32), ("in_h", C.c_int32), ("in_w", C.c_int32), ("in_c", C.c_int32),
                ("out_c", C.c_int32), ("kh", C.c_int32), ("kw", C.c_int32), ("stride", C.c_int32),
                ("act", C.c_int32)]


class AqNet(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("layers", C.POINTER(AqLayer)), ("head", C.c_int32),
                ("wscheme", C.c_int32), ("in_type", C.c_int32), ("qdenom", C.c_int32), ("ln_eps", C.c_float),
                ("wbits", C.c_int32)]


class AqRange(C.Structure):
    _fields_ = [("lo", C.c_float), ("hi", C.c_float)]


class AqExplore(C.Structure):
    _fields_ = [("seed", C.c_uint64), ("step", C.c_uint64), ("d_sigma", C.c_void_p), ("epsilon", C.c_float)]


class AqTaps(C.Structure):
    _fields_ = [("acc", C.POINTER(C.c_void_p)), ("act", C.POINTER(C.c_void_p)), ("ln_t", C.POINTER(C.c_void_p)),
                ("a0", C.c_void_p), ("y", C.c_void_p)]


class AqMatrix(C.Structure):
    _fields_ = [("d", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("ld", C.c_int64), ("dtype", C.c_int32)]


class AqBlocks(C.Structure):
    """aq_ckpt8 and aq_mx4, which are laid out alike."""
    _fields_ = [("d_codes", C.c_void_p), ("d_scales", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64)]


# The same as bytes, a third of the time of a Structure's construction and conversion (0.7 against 1.05 us a matrix; a small
# LayerNorm's two passes take five).  (The type as 64 bits: it and the padding behind it.)
_pack_matrix = struct.Struct("Pqqqq").pack
_pack_blocks = struct.Struct("PPqq").pack


class AqError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        msg = _lib.aq_status_string(status).decode() if _lib is not None else str(status)
        super().__init__(f"{where}: {msg} (aq_status {status})")


_lib = None


def load():
    """Loads libactorq.so; raises if it has not been built (no fallback path exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_1910_01055_amd.build`")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
    pp = C.POINTER(C.c_void_p)
    lib.aq_status_string.restype = C.c_char_p
    lib.aq_status_string.argtypes = [C.c_int]
    lib.aq_policy_create.argtypes = [C.POINTER(AqNet), C.POINTER(vp)]
    lib.aq_policy_destroy.argtypes = [vp]
    lib.aq_policy_reserve.argtypes = [vp, i64]
    lib.aq_policy_set_path.argtypes = [vp, i32]
    lib.aq_policy_status.argtypes = [vp, vp]
    lib.aq_policy_conv_stack_layers.argtypes = [vp, C.POINTER(C.c_int32)]
    lib.aq_policy_fp16_conv_stack_layers.argtypes = [vp, C.POINTER(C.c_int32)]
    lib.aq_policy_subbyte_layers.argtypes = [vp, i64, C.POINTER(C.c_int32)]
    lib.aq_policy_fused_plan.argtypes = [vp, i64, C.POINTER(C.c_int32), C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
    lib.aq_policy_fp32_plan.argtypes = [vp, i64, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
    lib.aq_policy_fp16_plan.argtypes = [vp, i64, C.POINTER(C.c_int32)]
    lib.aq_quantize_tensor.argtypes = [vp, i64, i64, i32, i32, vp, vp, vp, vp, vp]
    lib.aq_stream_reference.argtypes = [vp, i64, vp, vp]
    lib.aq_mfma_loop_reference.argtypes = [vp, vp, i32, i32, i32, vp, vp]
    lib.aq_quantize_params.argtypes = [vp, pp, pp, pp, pp, C.POINTER(AqRange), vp]
    lib.aq_policy_export_layer.argtypes = [vp, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.aq_policy_export_act_qparams.argtypes = [vp, vp, vp, vp]
    lib.aq_policy_forward_int8.argtypes = [vp, vp, i64, vp, C.POINTER(AqTaps), vp]
    lib.aq_policy_forward_int8_static.argtypes = [vp, vp, i64, vp, vp]
    lib.aq_policy_forward_fp32_params.argtypes = [vp, pp, pp, pp, pp, vp, i64, vp, vp, vp]
    lib.aq_policy_set_params_fp32.argtypes = [vp, pp, pp, pp, pp, vp]
    lib.aq_policy_forward_fp32.argtypes = [vp, vp, i64, vp, vp]
    lib.aq_calibrate_fp32.argtypes = [vp, vp, i64, C.POINTER(AqRange), vp]
    lib.aq_policy_blob_size.argtypes = [vp, C.POINTER(C.c_uint64)]
    lib.aq_policy_export_blob.argtypes = [vp, vp, C.c_uint64, vp]
    lib.aq_policy_import_blob.argtypes = [vp, vp, C.c_uint64, vp]
    lib.aq_policy_explore.argtypes = [vp, vp, i64, C.POINTER(AqExplore), vp]
    lib.aq_policy_step_int8.argtypes = [vp, vp, i64, vp, C.POINTER(AqExplore), C.POINTER(AqTaps), vp]
    lib.aq_policy_packed_blob_size.argtypes = [vp, C.POINTER(C.c_uint64)]
    lib.aq_policy_export_packed_blob.argtypes = [vp, vp, C.c_uint64, vp]
    lib.aq_policy_import_packed_blob.argtypes = [vp, vp, C.c_uint64, vp]
    lib.aq_convert_params_fp16.argtypes = [vp, pp, pp, pp, pp, vp]
    lib.aq_policy_forward_fp16.argtypes = [vp, vp, i64, vp, pp, vp]
    mat = blk = vp  # (packed bytes, or a structure by reference)
    u64, f32 = C.c_uint64, C.c_float
    lib.aq_layernorm_forward.argtypes = [mat, vp, vp, f32, mat, vp, vp, blk, vp]
    lib.aq_layernorm_backward.argtypes = [mat, mat, blk, vp, vp, vp, mat, vp, vp, vp, u64, vp]
    lib.aq_layernorm_backward_workspace.argtypes = [i64, i64, C.POINTER(u64)]
    lib.aq_ckpt8_pack.argtypes = lib.aq_mx4_quantize.argtypes = [mat, blk, vp]
    lib.aq_ckpt8_unpack.argtypes = lib.aq_mx4_dequantize.argtypes = [blk, mat, vp]
    lib.aq_ckpt8_weight_grad.argtypes = [mat, blk, mat, vp, vp, u64, vp]
    lib.aq_mx4_linear.argtypes = [mat, blk, vp, mat, vp, u64, vp]
    lib.aq_mx4_matmul.argtypes = [blk, blk, vp, mat, vp]
    lib.aq_mx4_input_grad.argtypes = [mat, blk, mat, vp, u64, vp]
    for name in ("aq_ckpt8_weight_grad_workspace", "aq_mx4_linear_workspace", "aq_mx4_input_grad_workspace"):
        getattr(lib, name).argtypes = [i64, i64, i64, C.POINTER(u64)]
    for name in EXPORTS:
        fn = getattr(lib, name)
        # (addresses travel as plain integers, which ctypes cuts to 32 bits where no argument types are declared)
        if fn.argtypes is None:
            raise RuntimeError(f"{name} has no argument types")
        if name != "aq_status_string":
            fn.restype = C.c_int
    _lib = lib
    return lib


def _first_stream():
    """The current stream as a raw handle; afterwards without building a torch.cuda.Stream object for every call,
    which took 2.7 of the 7.5 us that a small policy's forward took in all (the handle itself is 0.1 us)."""
    global _stream
    import torch
    handle = torch.cuda.current_stream().cuda_stream  # (initializes CUDA)
    device, raw = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
    _stream = lambda: raw(device())  # noqa: E731
    return handle


_stream = _first_stream


def _ptr(t):
    return None if t is None else t.data_ptr()


_PTR_ARRAYS = [C.c_void_p * n for n in range(MAX_LAYERS + 1)]
_RANGE_ARRAYS = [AqRange * n for n in range(MAX_LAYERS + 1)]


def _ptr_array(tensors, n):
    if tensors is None:
        return _PTR_ARRAYS[n]()
    return _PTR_ARRAYS[n](*[None if t is None else t.data_ptr() for t in tensors[:n]])


def _range_array(ranges, n):
    return _RANGE_ARRAYS[n](*[(float(lo), float(hi)) for lo, hi in ranges])


def _check(status, where):
    if status != OK:
        raise AqError(status, where)


def make_net(net: dict):
    """dict description (see synth.CONFIGS) -> (AqNet, keep-alive layer array)."""
    n = len(net["layers"])
    arr = (AqLayer * n)()
    for i, l in enumerate(net["layers"]):
        if l["kind"] == "fc":
            arr[i] = AqLayer(KIND["fc"], 1, 1, l["in"], l["out"], 1, 1, 1, ACT[l["act"]])
        else:
            arr[i] = AqLayer(KIND["conv"], l["in_h"], l["in_w"], l["in_c"], l["out_c"], l["kh"], l["kw"],
                             l["stride"], ACT[l["act"]])
    cnet = AqNet(n, arr, HEAD[net["head"]], WSCHEME[net["wscheme"]], INTYPE[net["in_type"]], int(net["qdenom"]),
                 float(net["ln_eps"]), int(net.get("wbits", 0)))
    return cnet, arr


class Policy:
    """Owns one aq_policy handle.  Methods carry the C entry points' names."""

    def __init__(self, net: dict):
        lib = load()
        self.net = net
        self.n_layers = len(net["layers"])
        cnet, keep = make_net(net)
        h = C.c_void_p()
        _check(lib.aq_policy_create(C.byref(cnet), C.byref(h)), "aq_policy_create")
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            load().aq_policy_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def policy_reserve(self, max_batch):
        _check(load().aq_policy_reserve(self._h, int(max_batch)), "aq_policy_reserve")

    def policy_set_path(self, path):
        _check(load().aq_policy_set_path(self._h, int(path)), "aq_policy_set_path")

    def policy_conv_stack_layers(self):
        n = C.c_int32(0)
        _check(load().aq_policy_conv_stack_layers(self._h, C.byref(n)), "aq_policy_conv_stack_layers")
        return int(n.value)

    def policy_fp16_conv_stack_layers(self):
        n = C.c_int32(0)
        _check(load().aq_policy_fp16_conv_stack_layers(self._h, C.byref(n)), "aq_policy_fp16_conv_stack_layers")
        return int(n.value)

    def policy_fused_plan(self, batch):
        """(rows per workgroup, feature tiles per wavefront, kernel: 0 general / 1 pipelined for wide layers /
        2 the kernel for small networks) of the fused launch at this batch; (0, 0, 0) = one launch per layer."""
        r, t, w = C.c_int32(0), C.c_int32(0), C.c_int32(0)
        _check(load().aq_policy_fused_plan(self._h, int(batch), C.byref(r), C.byref(t), C.byref(w)), "aq_policy_fused_plan")
        return int(r.value), int(t.value), int(w.value)

    def policy_fp32_plan(self, batch):
        """(rows per workgroup of the whole-policy launch or 0, per layer (features, rows) of its tile where each layer
        has a launch of its own) of the fp32 actor at this batch."""
        r, t = C.c_int32(0), (C.c_int32 * (2 * self.n_layers))()
        _check(load().aq_policy_fp32_plan(self._h, int(batch), C.byref(r), t), "aq_policy_fp32_plan")
        return int(r.value), [] if r.value else list(zip(t[::2], t[1::2]))

    def policy_fp16_plan(self, batch):
        """Rows per workgroup of the half-precision actor's whole-policy launch at this batch; 0 = a launch per layer."""
        r = C.c_int32(0)
        _check(load().aq_policy_fp16_plan(self._h, int(batch), C.byref(r)), "aq_policy_fp16_plan")
        return int(r.value)

    def policy_subbyte_layers(self, batch):
        """Layers of a forward pass at this batch that stream their weights as nibbles (policies of <= 4 bits)."""
        n = C.c_int32(0)
        _check(load().aq_policy_subbyte_layers(self._h, int(batch), C.byref(n)), "aq_policy_subbyte_layers")
        return int(n.value)

    def policy_status(self):
        return load().aq_policy_status(self._h, _stream())

    def policy_step_int8(self, obs, actions, seed, step, sigma=None, epsilon=0.0):
        """8-bit forward plus exploration in one call (fused into the forward kernel where possible)."""
        ex = AqExplore(int(seed), int(step), 0 if sigma is None else sigma.data_ptr(), float(epsilon))
        _check(load().aq_policy_step_int8(self._h, _ptr(obs), obs.shape[0], _ptr(actions), C.byref(ex), None,
                                          _stream()), "aq_policy_step_int8")

    def policy_explore(self, actions, seed, step, sigma=None, epsilon=0.0):
        """In place on the actions of a forward: Gaussian noise with per-row sigma (device fp32 [batch]) for
        continuous heads, epsilon-greedy for argmax heads."""
        ex = AqExplore(int(seed), int(step), 0 if sigma is None else sigma.data_ptr(), float(epsilon))
        _check(load().aq_policy_explore(self._h, _ptr(actions), actions.shape[0], C.byref(ex), _stream()),
               "aq_policy_explore")

    def policy_blob_size(self):
        n = C.c_uint64(0)
        _check(load().aq_policy_blob_size(self._h, C.byref(n)), "aq_policy_blob_size")
        return int(n.value)

    def policy_export_blob(self, blob):
        """blob: a uint8 device tensor of at least policy_blob_size() bytes."""
        _check(load().aq_policy_export_blob(self._h, _ptr(blob), blob.numel() * blob.element_size(), _stream()),
               "aq_policy_export_blob")

    def policy_import_blob(self, blob):
        _check(load().aq_policy_import_blob(self._h, _ptr(blob), blob.numel() * blob.element_size(), _stream()),
               "aq_policy_import_blob")

    def policy_packed_blob_size(self):
        n = C.c_uint64(0)
        _check(load().aq_policy_packed_blob_size(self._h, C.byref(n)), "aq_policy_packed_blob_size")
        return int(n.value)

    def policy_export_packed_blob(self, blob):
        _check(load().aq_policy_export_packed_blob(self._h, _ptr(blob), blob.numel() * blob.element_size(), _stream()),
               "aq_policy_export_packed_blob")

    def policy_import_packed_blob(self, blob):
        _check(load().aq_policy_import_packed_blob(self._h, _ptr(blob), blob.numel() * blob.element_size(), _stream()),
               "aq_policy_import_packed_blob")

    def quantize_params(self, w, b, gamma, beta, ranges):
        """w, b, gamma, beta: per-layer lists of device tensors (entries or lists may be None);
        ranges: n_layers (lo, hi) pairs."""
        n = self.n_layers
        r = _range_array(ranges, n)
        _check(load().aq_quantize_params(self._h, _ptr_array(w, n), _ptr_array(b, n), _ptr_array(gamma, n),
                                         _ptr_array(beta, n), r, _stream()), "aq_quantize_params")

    def policy_export_layer(self, layer, codes=None, w_scale=None, w_zp=None, bias_q=None, mult=None, rshift=None,
                            m=None):
        _check(load().aq_policy_export_layer(self._h, int(layer), _ptr(codes), _ptr(w_scale), _ptr(w_zp),
                                             _ptr(bias_q), _ptr(mult), _ptr(rshift), _ptr(m), _stream()),
               "aq_policy_export_layer")

    def policy_export_act_qparams(self, scale, zp):
        _check(load().aq_policy_export_act_qparams(self._h, _ptr(scale), _ptr(zp), _stream()),
               "aq_policy_export_act_qparams")

    def policy_forward_int8(self, obs, actions, taps=None):
        """taps: dict with optional keys acc/act/ln_t (per-layer lists of tensors or None), a0, y."""
        batch = obs.shape[0]
        ctaps = None
        if taps:
            n = self.n_layers
            keep = [_ptr_array(taps.get(k), n) for k in ("acc", "act", "ln_t")]
            ctaps = AqTaps(C.cast(keep[0], C.POINTER(C.c_void_p)), C.cast(keep[1], C.POINTER(C.c_void_p)),
                           C.cast(keep[2], C.POINTER(C.c_void_p)), _ptr(taps.get("a0")), _ptr(taps.get("y")))
        _check(load().aq_policy_forward_int8(self._h, _ptr(obs), batch, _ptr(actions),
                                             C.byref(ctaps) if ctaps is not None else None, _stream()),
               "aq_policy_forward_int8")

    def policy_forward_int8_static(self, obs, actions):
        """The 8-bit forward that allocates nothing (scratch in the library's static device buffer)."""
        _check(load().aq_policy_forward_int8_static(self._h, _ptr(obs), obs.shape[0], _ptr(actions), _stream()),
               "aq_policy_forward_int8_static")

    def policy_forward_fp32_params(self, w, b, gamma, beta, obs, actions, ranges_out=None):
        n = self.n_layers
        _check(load().aq_policy_forward_fp32_params(self._h, _ptr_array(w, n), _ptr_array(b, n), _ptr_array(gamma, n),
                                                    _ptr_array(beta, n), _ptr(obs), obs.shape[0], _ptr(actions),
                                                    _ptr(ranges_out), _stream()), "aq_policy_forward_fp32_params")

    def policy_set_params_fp32(self, w, b, gamma, beta):
        n = self.n_layers
        _check(load().aq_policy_set_params_fp32(self._h, _ptr_array(w, n), _ptr_array(b, n), _ptr_array(gamma, n),
                                                _ptr_array(beta, n), _stream()), "aq_policy_set_params_fp32")

    def policy_forward_fp32(self, obs, actions):
        _check(load().aq_policy_forward_fp32(self._h, _ptr(obs), obs.shape[0], _ptr(actions), _stream()),
               "aq_policy_forward_fp32")

    def calibrate_fp32(self, obs):
        """(min, max) per activation tensor over this batch, as a list of n_layers pairs (waits for the stream)."""
        r = _RANGE_ARRAYS[self.n_layers]()
        _check(load().aq_calibrate_fp32(self._h, _ptr(obs), obs.shape[0], r, _stream()), "aq_calibrate_fp32")
        return [(float(x.lo), float(x.hi)) for x in r]

    def quantize_kept_params(self, ranges):
        """aq_quantize_params on the parameters kept by policy_set_params_fp32 (NULL parameter arrays)."""
        n = self.n_layers
        r = _range_array(ranges, n)
        _check(load().aq_quantize_params(self._h, None, None, None, None, r, _stream()), "aq_quantize_params")

    def convert_params_fp16(self, w, b, gamma, beta):
        n = self.n_layers
        _check(load().aq_convert_params_fp16(self._h, _ptr_array(w, n), _ptr_array(b, n), _ptr_array(gamma, n),
                                             _ptr_array(beta, n), _stream()), "aq_convert_params_fp16")

    def policy_forward_fp16(self, obs, actions, taps_out=None):
        taps = _ptr_array(taps_out, self.n_layers) if taps_out is not None else None
        _check(load().aq_policy_forward_fp16(self._h, _ptr(obs), obs.shape[0], _ptr(actions), taps, _stream()),
               "aq_policy_forward_fp16")


def to_dev(a, device="cuda:0"):
    """numpy array (or None) -> contiguous device tensor (or None): device memory plumbing only."""
    import numpy as np
    import torch
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(device)


def upload_params(params, device="cuda:0"):
    """Per-layer fp32 parameters (dicts with w, b, optional gamma, beta) -> four lists of device tensors."""
    return ([to_dev(p["w"], device) for p in params], [to_dev(p["b"], device) for p in params],
            [to_dev(p.get("gamma"), device) for p in params], [to_dev(p.get("beta"), device) for p in params])


def stream_reference(src, n, dst):
    _check(load().aq_stream_reference(_ptr(src), int(n), _ptr(dst), _stream()), "aq_stream_reference")


def mfma_loop_reference(weights, acts, ksteps, stream_weights, workgroups, acc):
    _check(load().aq_mfma_loop_reference(_ptr(weights), _ptr(acts), int(ksteps), int(bool(stream_weights)), int(workgroups),
                                         _ptr(acc), _stream()), "aq_mfma_loop_reference")


def quantize_tensor(w, rows, cols, wscheme, qdenom, codes, scale, zp, workspace):
    _check(load().aq_quantize_tensor(_ptr(w), int(rows), int(cols), WSCHEME[wscheme], int(qdenom), _ptr(codes),
                                     _ptr(scale), _ptr(zp), _ptr(workspace), _stream()), "aq_quantize_tensor")


# ---- the learner's operators.  Matrices are two-dimensional device tensors whose rows are contiguous (any distance between rows);
# vectors are contiguous fp32 tensors; `workspace` is a uint8 tensor of the size that the matching *_workspace call gives (None for 0).
# Tensors in ordinary host memory, whose addresses fault the GPU, are refused: 0.05 us a tensor, which the calls save where they ask less of
# Python otherwise (`_lib or load()`).

_DTYPES = {}
_F32 = None


def _learn_dtypes():
    global _F32
    import torch
    _F32 = torch.float32
    _DTYPES.update({torch.float32: 0, torch.float16: 1, torch.bfloat16: 2})


def _reachable(*tensors):
    """Refuses tensors that the GPU does not reach (callers ask is_cuda first; this is for pinned memory and the refusal)."""
    for t in tensors:
        if not t.is_cuda and t.numel() and not t.is_pinned():
            raise ValueError("a tensor lies in host memory that the GPU does not reach")


def _matrix(t):
    """A tensor as an aq_matrix."""
    try:
        rows, cols = t.shape
        dtype = _DTYPES[t.dtype]
    except (ValueError, KeyError):
        if _F32 is None:
            _learn_dtypes()
            return _matrix(t)
        raise ValueError("a matrix is a two-dimensional tensor of float32, float16 or bfloat16") from None
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError("the values of a row are contiguous")
    return _pack_matrix(t.data_ptr(), rows, cols, ld if rows > 1 else cols, dtype)


def _vector(t, n, what):
    """A contiguous fp32 vector of n values as a pointer; None stays None."""
    if t is None:
        return None
    if t.dtype is not _F32 or t.numel() != n or not t.is_contiguous():
        if _F32 is None:
            _learn_dtypes()
            return _vector(t, n, what)
        raise ValueError(f"{what} is a contiguous float32 tensor of {n} values")
    if not t.is_cuda:
        _reachable(t)
    return t.data_ptr()


def _bytes(workspace):
    """The size of a workspace."""
    size = 0 if workspace is None else workspace.nbytes
    if size:
        if not workspace.is_contiguous():  # (a tensor that repeats values has fewer bytes than it counts)
            raise ValueError("a workspace is contiguous")
        if not workspace.is_cuda:
            _reachable(workspace)
    return size


class _Blocks:
    """Codes and scales of a [rows][cols] tensor in blocks of 32 values along a row."""
    CODE_BYTES = 0  # of a block

    def __init__(self, codes, scales, cols):
        import torch
        rows, blocks = scales.shape
        if blocks != (cols + 31) // 32 or tuple(codes.shape) != (rows, self.CODE_BYTES * blocks):
            raise ValueError(f"codes are [rows][{self.CODE_BYTES} B] and scales [rows][B], B = ceil(cols / 32)")
        if scales.dtype != torch.uint8 or codes.element_size() != 1 or not codes.is_contiguous() or not scales.is_contiguous():
            raise ValueError("codes and scales are contiguous tensors of bytes")
        self.__dict__.update(codes=codes, scales=scales, rows=rows, cols=int(cols), _near=codes.is_cuda and scales.is_cuda,
                             _c=_pack_blocks(codes.data_ptr(), scales.data_ptr(), rows, int(cols)))

    def __setattr__(self, name, value):
        raise AttributeError(f"{name}: blocks of other tensors are made anew, as calls are handed these tensors' addresses")


class Ckpt8(_Blocks):
    """An 8-bit checkpoint (aq_ckpt8): codes int8 [rows][32 B], scales uint8 [rows][B], B = ceil(cols / 32)."""
    CODE_BYTES = 32


class Mx4(_Blocks):
    """A microscaled 4-bit tensor (aq_mx4): codes uint8 [rows][16 B], scales uint8 [rows][B], B = ceil(cols / 32)."""
    CODE_BYTES = 16


def _kept(q):
    """A Ckpt8 as an aq_ckpt8; whatever else would be taken for one of its sizes."""
    if isinstance(q, Ckpt8):
        if not q._near:
            _reachable(q.codes, q.scales)
        return q._c
    raise ValueError("an 8-bit checkpoint is a Ckpt8")


def _mx4(q):
    """An Mx4 as an aq_mx4."""
    if isinstance(q, Mx4):
        if not q._near:
            _reachable(q.codes, q.scales)
        return q._c
    raise ValueError("a 4-bit tensor is an Mx4")


def _blocks_empty(kind, code_type, rows, cols, device):
    import torch
    b = (int(cols) + 31) // 32
    return kind(torch.empty(int(rows), kind.CODE_BYTES * b, dtype=code_type, device=device),
                torch.empty(int(rows), b, dtype=torch.uint8, device=device), cols)


def ckpt8_empty(rows, cols, device="cuda:0"):
    import torch
    return _blocks_empty(Ckpt8, torch.int8, rows, cols, device)


def mx4_empty(rows, cols, device="cuda:0"):
    import torch
    return _blocks_empty(Mx4, torch.uint8, rows, cols, device)


def _size(fn, *sizes):
    n = C.c_uint64(0)
    _check(getattr(load(), fn)(*[int(v) for v in sizes], C.byref(n)), fn)
    return int(n.value)


def layernorm_backward_workspace(rows, cols):
    return _size("aq_layernorm_backward_workspace", rows, cols)


def ckpt8_weight_grad_workspace(rows, n, k):
    return _size("aq_ckpt8_weight_grad_workspace", rows, n, k)


def mx4_linear_workspace(rows, n, k):
    return _size("aq_mx4_linear_workspace", rows, n, k)


def mx4_input_grad_workspace(rows, n, k):
    return _size("aq_mx4_input_grad_workspace", rows, n, k)


def layernorm_forward(x, gamma, beta, eps, y, mean=None, rstd=None, kept=None):
    """y = LayerNorm(x); kept: a Ckpt8 that receives x."""
    rows, cols = x.shape
    if not (x.is_cuda and y.is_cuda):
        _reachable(x, y)
    status = (_lib or load()).aq_layernorm_forward(_matrix(x), _vector(gamma, cols, "gamma"), _vector(beta, cols, "beta"), eps, _matrix(y),
                                                   _vector(mean, rows, "mean"), _vector(rstd, rows, "rstd"),
                                                   None if kept is None else _kept(kept), _stream())
    if status:
        raise AqError(status, "aq_layernorm_forward")


def layernorm_backward(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, workspace=None):
    """x: the forward pass's input, or its Ckpt8."""
    rows, cols = dy.shape
    blocks = isinstance(x, _Blocks)
    if not (dy.is_cuda and dx.is_cuda and (blocks or x.is_cuda)):
        _reachable(dy, dx, dy if blocks else x)
    status = (_lib or load()).aq_layernorm_backward(_matrix(dy), None if blocks else _matrix(x), _kept(x) if blocks else None,
                                                    _vector(gamma, cols, "gamma"), _vector(mean, rows, "mean"), _vector(rstd, rows, "rstd"),
                                                    _matrix(dx), _vector(dgamma, cols, "dgamma"), _vector(dbeta, cols, "dbeta"),
                                                    _ptr(workspace), _bytes(workspace), _stream())
    if status:
        raise AqError(status, "aq_layernorm_backward")


def ckpt8_pack(x, kept):
    if not x.is_cuda:
        _reachable(x)
    status = (_lib or load()).aq_ckpt8_pack(_matrix(x), _kept(kept), _stream())
    if status:
        raise AqError(status, "aq_ckpt8_pack")


def ckpt8_unpack(kept, x):
    if not x.is_cuda:
        _reachable(x)
    status = (_lib or load()).aq_ckpt8_unpack(_kept(kept), _matrix(x), _stream())
    if status:
        raise AqError(status, "aq_ckpt8_unpack")


def ckpt8_weight_grad(dy, kept, dw, db=None, workspace=None):
    if not (dy.is_cuda and dw.is_cuda):
        _reachable(dy, dw)
    status = (_lib or load()).aq_ckpt8_weight_grad(_matrix(dy), _kept(kept), _matrix(dw), _vector(db, dy.shape[1], "db"), _ptr(workspace),
                                                   _bytes(workspace), _stream())
    if status:
        raise AqError(status, "aq_ckpt8_weight_grad")


def mx4_quantize(x, q):
    if not x.is_cuda:
        _reachable(x)
    status = (_lib or load()).aq_mx4_quantize(_matrix(x), _mx4(q), _stream())
    if status:
        raise AqError(status, "aq_mx4_quantize")


def mx4_dequantize(q, x):
    if not x.is_cuda:
        _reachable(x)
    status = (_lib or load()).aq_mx4_dequantize(_mx4(q), _matrix(x), _stream())
    if status:
        raise AqError(status, "aq_mx4_dequantize")


def mx4_linear(x, w, bias, y, workspace=None):
    """y = Q(x) w^T + bias; w: Mx4 [n][k]."""
    if not (x.is_cuda and y.is_cuda):
        _reachable(x, y)
    status = (_lib or load()).aq_mx4_linear(_matrix(x), _mx4(w), _vector(bias, w.rows, "bias"), _matrix(y), _ptr(workspace),
                                            _bytes(workspace), _stream())
    if status:
        raise AqError(status, "aq_mx4_linear")


def mx4_matmul(x, w, bias, y):
    """The same from an Mx4 x."""
    if not y.is_cuda:
        _reachable(y)
    status = (_lib or load()).aq_mx4_matmul(_mx4(x), _mx4(w), _vector(bias, w.rows, "bias"), _matrix(y), _stream())
    if status:
        raise AqError(status, "aq_mx4_matmul")


def mx4_input_grad(dy, w, dx, workspace=None):
    """dx = dy w; w: Mx4 [n][k]."""
    if not (dy.is_cuda and dx.is_cuda):
        _reachable(dy, dx)
    status = (_lib or load()).aq_mx4_input_grad(_matrix(dy), _mx4(w), _matrix(dx), _ptr(workspace), _bytes(workspace), _stream())
    if status:
        raise AqError(status, "aq_mx4_input_grad")
