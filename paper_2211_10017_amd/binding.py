"""Thin ctypes binding of the C-ABI HIP library (include/moe_wq.h).

Argument marshalling only: every function takes torch CUDA tensors, checks their dtype,
device and contiguity, and passes raw device pointers plus the current stream.  No step of
the layer runs in Python or in torch ops.  If the library has not been built the first call
raises: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmoe_wq.so")

MOE_F16, MOE_BF16, MOE_F32 = 0, 1, 2
_DT = {torch.float16: MOE_F16, torch.bfloat16: MOE_BF16, torch.float32: MOE_F32}

EXPORTS = ["moe_last_error", "moe_last_ffn_kernels", "moe_device_info", "moe_abi_version", "moe_quantize_experts", "moe_gate_topk",
           "moe_permute_workspace_bytes", "moe_permute", "moe_grouped_ffn_wq_workspace_bytes",
           "moe_grouped_ffn_wq", "moe_combine", "moe_pack_fp16_experts", "moe_grouped_gemm_wq",
           "moe_grouped_ffn_wq_routed_supported", "moe_grouped_ffn_wq_routed", "moe_grouped_ffn_wq_indexed", "moe_grouped_ffn_wq_indexed_pays",
           "moe_grouped_ffn_wq_unsorted_supported", "moe_grouped_ffn_wq_unsorted_pays", "moe_grouped_ffn_wq_unsorted",
           "moe_grouped_ffn_wq_gated_supported", "moe_grouped_ffn_wq_gated_pays", "moe_grouped_ffn_wq_gated",
           "moe_grouped_ffn_wq_sliced_workspace_bytes", "moe_grouped_ffn_wq_sliced_pays", "moe_grouped_ffn_wq_sliced",
           "moe_grouped_ffn_wq_noalloc_max_bytes", "moe_grouped_ffn_wq_noalloc",
           "moe_mx4_quantize_rows", "moe_mx4_quantize_experts", "moe_mx4_dequantize", "moe_grouped_gemm_mx4",
           "moe_grouped_ffn_mx4_workspace_bytes", "moe_grouped_ffn_mx4",
           "moe_balance_loss_workspace_bytes", "moe_balance_loss", "moe_balance_loss_backward"]

LAYER_MAX_EXPERTS = 256   # experts of a whole layer call: moe_gate_topk's limit (moe_permute: 1024, the FFN: 4096)

_lib = None
ACTIVATIONS = {"relu": 0, "gelu": 1}     # MOE_ACT_RELU, MOE_ACT_GELU


class MoeError(RuntimeError):
    pass


def load():
    """Load libmoe_wq.so (once) and declare the signatures of include/moe_wq.h."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise MoeError("HIP library %s is missing: build it with "
                       "`python -m paper_2211_10017_amd.build` (no fallback exists)" % LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    vp, i, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    lib.moe_last_error.restype = ctypes.c_char_p
    lib.moe_last_error.argtypes = []
    lib.moe_last_ffn_kernels.restype = ctypes.c_char_p
    lib.moe_last_ffn_kernels.argtypes = []
    lib.moe_device_info.restype = i
    lib.moe_device_info.argtypes = [ctypes.POINTER(i)] * 4
    lib.moe_abi_version.restype = i
    lib.moe_quantize_experts.restype = i
    lib.moe_quantize_experts.argtypes = [vp, i, i, i, i, i, vp, vp, vp, vp]
    lib.moe_gate_topk.restype = i
    lib.moe_gate_topk.argtypes = [vp, i, vp, vp, vp, i, i, i, i, i, vp, vp, vp]
    lib.moe_permute_workspace_bytes.restype = sz
    lib.moe_permute_workspace_bytes.argtypes = [i, i, i]
    lib.moe_permute.restype = i
    lib.moe_permute.argtypes = [vp, vp, i, i, i, i, i, vp, vp, vp, vp, vp, sz, vp]
    lib.moe_grouped_ffn_wq_workspace_bytes.restype = sz
    lib.moe_grouped_ffn_wq_workspace_bytes.argtypes = [i, i, i, i, i]
    lib.moe_grouped_ffn_wq.restype = i
    lib.moe_grouped_ffn_wq.argtypes = [vp, i, vp, i, i, i, i, i, i, i, i, vp, vp, vp, vp, vp, vp, vp, i, vp, sz, vp]
    lib.moe_grouped_ffn_wq_noalloc_max_bytes.restype = sz
    lib.moe_grouped_ffn_wq_noalloc_max_bytes.argtypes = []
    lib.moe_grouped_ffn_wq_noalloc.restype = i
    lib.moe_grouped_ffn_wq_noalloc.argtypes = [vp, i, vp, i, i, i, i, i, i, i, i, vp, vp, vp, vp, vp, vp, vp, i, vp]
    lib.moe_grouped_ffn_wq_routed_supported.restype = i
    lib.moe_grouped_ffn_wq_routed_supported.argtypes = [i, i, i, i, i, i, i, i]
    lib.moe_grouped_ffn_wq_routed.restype = i
    lib.moe_grouped_ffn_wq_routed.argtypes = [vp, i, vp, i, vp, vp, i, i, i, i, i, i, i, i, vp, vp, vp, vp, vp, vp, vp, i,
                                              vp, sz, vp]
    lib.moe_grouped_ffn_wq_indexed.restype = i
    lib.moe_grouped_ffn_wq_indexed.argtypes = [vp, i, vp, i, vp, vp, i, i, i, i, i, i, i, i, vp, vp, vp, vp, vp, vp, vp, i,
                                              vp, sz, vp]
    lib.moe_grouped_ffn_wq_indexed_pays.restype = i
    lib.moe_grouped_ffn_wq_indexed_pays.argtypes = [i, i, i, i, i, i, i, i]
    lib.moe_grouped_ffn_wq_unsorted_supported.restype = i
    lib.moe_grouped_ffn_wq_unsorted_supported.argtypes = [i, i, i, i, i, i, i, i]
    lib.moe_grouped_ffn_wq_unsorted_pays.restype = i
    lib.moe_grouped_ffn_wq_unsorted_pays.argtypes = [i, i, i, i, i, i, i, i]
    lib.moe_grouped_ffn_wq_unsorted.restype = i
    lib.moe_grouped_ffn_wq_unsorted.argtypes = [vp, i, vp, vp, i, i, i, i, i, i, i, i, vp, vp, vp, vp, vp, vp, vp, i, vp, vp, vp,
                                                vp, sz, vp]
    lib.moe_grouped_ffn_wq_gated_supported.restype = i
    lib.moe_grouped_ffn_wq_gated_supported.argtypes = [i, i, i, i, i, i, i, i]
    lib.moe_grouped_ffn_wq_gated_pays.restype = i
    lib.moe_grouped_ffn_wq_gated_pays.argtypes = [i, i, i, i, i, i, i, i]
    lib.moe_grouped_ffn_wq_gated.restype = i
    lib.moe_grouped_ffn_wq_gated.argtypes = [vp, i, vp, vp, i, i, i, i, i, i, i, i, vp, vp, vp, vp, vp, vp, vp, i, vp, vp, vp,
                                             vp, sz, vp]
    lib.moe_grouped_ffn_wq_sliced_workspace_bytes.restype = sz
    lib.moe_grouped_ffn_wq_sliced_workspace_bytes.argtypes = [i, i, i, i, i, i, i, i]
    lib.moe_grouped_ffn_wq_sliced_pays.restype = i
    lib.moe_grouped_ffn_wq_sliced_pays.argtypes = [i, i, i, i, i, i, i, i]
    lib.moe_grouped_ffn_wq_sliced.restype = i
    lib.moe_grouped_ffn_wq_sliced.argtypes = [vp, i, vp, vp, i, i, i, i, i, i, i, i, vp, vp, vp, vp, vp, vp, vp, i, vp, vp, vp,
                                              vp, sz, vp]
    lib.moe_pack_fp16_experts.restype = i
    lib.moe_pack_fp16_experts.argtypes = [vp, i, i, i, vp, vp]
    lib.moe_grouped_gemm_wq.restype = i
    lib.moe_grouped_gemm_wq.argtypes = [vp, vp, i, i, i, i, i, i, i, vp, vp, vp, i, vp]
    lib.moe_combine.restype = i
    lib.moe_combine.argtypes = [vp, i, vp, vp, vp, i, i, i, vp, i, vp]
    i64, f = ctypes.c_int64, ctypes.c_float
    lib.moe_mx4_quantize_rows.restype = i
    lib.moe_mx4_quantize_rows.argtypes = [vp, i, i, i, i64, vp, vp, vp]
    lib.moe_mx4_quantize_experts.restype = i
    lib.moe_mx4_quantize_experts.argtypes = [vp, i, i, i, vp, vp, vp]
    lib.moe_mx4_dequantize.restype = i
    lib.moe_mx4_dequantize.argtypes = [vp, vp, i, i, i, vp, i, vp]
    lib.moe_grouped_gemm_mx4.restype = i
    lib.moe_grouped_gemm_mx4.argtypes = [vp, vp, i, vp, i, vp, i, i, i, i, i, vp, vp, vp, i, vp, i, vp]
    lib.moe_grouped_ffn_mx4_workspace_bytes.restype = sz
    lib.moe_grouped_ffn_mx4_workspace_bytes.argtypes = [i, i, i, i]
    lib.moe_grouped_ffn_mx4.restype = i
    lib.moe_grouped_ffn_mx4.argtypes = [vp, i, i, vp, i, vp, i, i, i, i, i, i, vp, vp, vp, vp, vp, vp, vp, i, vp, sz, vp]
    lib.moe_balance_loss_workspace_bytes.restype = sz
    lib.moe_balance_loss_workspace_bytes.argtypes = [i, i]
    lib.moe_balance_loss.restype = i
    lib.moe_balance_loss.argtypes = [vp, i, vp, i, i, i, i, f, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.moe_balance_loss_backward.restype = i
    lib.moe_balance_loss_backward.argtypes = [vp, i, vp, i, i, i, i, vp, vp, vp, vp, vp]
    _lib = lib
    return lib


def moe_device_info() -> dict:
    """Compute units, engine / memory clock (kHz) and memory bus width (bits) of the current device."""
    v = [ctypes.c_int(0) for _ in range(4)]
    _check(load().moe_device_info(*[ctypes.byref(x) for x in v]), "moe_device_info")
    return dict(zip(("compute_units", "engine_clock_khz", "memory_clock_khz", "memory_bus_bits"), (x.value for x in v)))


def _check(rc: int, what: str):
    if rc != 0:
        raise MoeError("%s failed (code %d): %s" % (what, rc, load().moe_last_error().decode()))


def _ptr(t, dtype=None, name="tensor"):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise MoeError("%s must be a contiguous CUDA tensor" % name)
    if dtype is not None and t.dtype is not dtype and not (isinstance(dtype, tuple) and t.dtype in dtype):
        raise MoeError("%s has dtype %s, expected %s" % (name, t.dtype, dtype))
    return t.data_ptr()


# What torch.cuda.current_stream() itself calls; not part of torch's interface, so a torch without them takes the long way.
_raw_stream, _raw_device = (getattr(torch._C, name, None) for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))


def current_stream_handle() -> int:
    """torch.cuda.current_stream().cuda_stream without the Stream object around it, whose making takes 2.5 us: a call of one token is three
    launches of 3 us each on the host and hardly more on the device (host time of a step 14.0 -> 10.4 us, the step 14.24 -> 13.96)."""
    if _raw_stream is None or _raw_device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_raw_device())


def _stream():
    return current_stream_handle()


def moe_quantize_experts(w, bits: int, group_size: int = 0, want_canon: bool = True,
                         want_packed: bool = True):
    """w fp32 [E,K,N] -> (q_canon uint8/int8, scales fp16 [E,K/g,N], q_packed uint8)."""
    E, K, N = w.shape
    g = K if group_size in (0, K) else group_size
    dev = w.device
    nbytes = E * K * N * bits // 8
    q_canon = None
    if want_canon:
        q_canon = (torch.empty((E, K, N), dtype=torch.int8, device=dev) if bits == 8
                   else torch.empty((E, K, N // 2), dtype=torch.uint8, device=dev))
    scales = torch.empty((E, K // g, N), dtype=torch.float16, device=dev)
    q_packed = torch.empty(nbytes, dtype=torch.uint8, device=dev) if want_packed else None
    rc = load().moe_quantize_experts(_ptr(w, torch.float32, "w"), E, K, N, bits, group_size,
                                     _ptr(q_canon), _ptr(scales), _ptr(q_packed), _stream())
    _check(rc, "moe_quantize_experts")
    return q_canon, scales, q_packed


def moe_quantize_experts_into(w, bits, group_size, q_canon, scales, q_packed):
    """Same call writing into caller-provided slices (for expert-at-a-time quantisation)."""
    E, K, N = w.shape
    rc = load().moe_quantize_experts(_ptr(w, torch.float32, "w"), E, K, N, bits, group_size,
                                     _ptr(q_canon), _ptr(scales, torch.float16), _ptr(q_packed), _stream())
    _check(rc, "moe_quantize_experts")


def moe_gate_topk(x, wg, bias, k: int, renormalize: bool = True, out=None, finished=None):
    T, d = x.shape
    E = wg.shape[1]
    if wg.dtype != x.dtype or wg.shape[0] != d:
        raise MoeError("wg must be [d,E] in the dtype of x")
    if out is None:
        idx = torch.empty((T, k), dtype=torch.int32, device=x.device)
        scale = torch.empty((T, k), dtype=torch.float32, device=x.device)
    else:
        idx, scale = out
    rc = load().moe_gate_topk(_ptr(x, (torch.float16, torch.bfloat16), "x"), _DT[x.dtype], _ptr(wg),
                              _ptr(bias, torch.float32, "bias"), _ptr(finished, torch.uint8, "finished"),
                              T, d, E, k, int(renormalize),
                              _ptr(idx, torch.int32), _ptr(scale, torch.float32), _stream())
    _check(rc, "moe_gate_topk")
    return idx, scale


def moe_permute_workspace_bytes(T: int, k: int, E: int) -> int:
    return int(load().moe_permute_workspace_bytes(T, k, E))


def moe_permute(expert_idx, x, E: int, out=None, workspace=None):
    T, k = expert_idx.shape
    d = x.shape[1]
    R = T * k
    dev = x.device
    if out is None:
        x_perm = torch.empty((R, d), dtype=x.dtype, device=dev)
        perm_src = torch.empty(R, dtype=torch.int32, device=dev)
        inv_perm = torch.empty(R, dtype=torch.int32, device=dev)
        offsets = torch.empty(E + 1, dtype=torch.int32, device=dev)
    else:
        x_perm, perm_src, inv_perm, offsets = out
    if workspace is None:
        workspace = torch.empty(moe_permute_workspace_bytes(T, k, E), dtype=torch.uint8, device=dev)
    rc = load().moe_permute(_ptr(expert_idx, torch.int32, "expert_idx"), _ptr(x), _DT[x.dtype], T, k, E, d,
                            _ptr(x_perm), _ptr(perm_src, torch.int32), _ptr(inv_perm, torch.int32),
                            _ptr(offsets, torch.int32), _ptr(workspace), workspace.numel(), _stream())
    _check(rc, "moe_permute")
    return x_perm, perm_src, inv_perm, offsets


def moe_permute_index(expert_idx, E: int, d: int, act_dtype, perm_src, inv_perm, expert_offsets, workspace):
    """moe_permute without the copy of the rows, into buffers of the caller's."""
    T, k = expert_idx.shape
    if perm_src.numel() < T * k or inv_perm.numel() < T * k or expert_offsets.numel() < E + 1:
        raise MoeError("perm_src and inv_perm must hold %d numbers and expert_offsets %d" % (T * k, E + 1))
    rc = load().moe_permute(_ptr(expert_idx, torch.int32, "expert_idx"), None, _DT[act_dtype], T, k, E, d, None, _ptr(perm_src, torch.int32, "perm_src"),
                            _ptr(inv_perm, torch.int32, "inv_perm"), _ptr(expert_offsets, torch.int32, "expert_offsets"), _ptr(workspace, torch.uint8, "workspace"), workspace.numel(), _stream())
    _check(rc, "moe_permute")


def moe_grouped_ffn_wq_workspace_bytes(R: int, d: int, F: int, E: int, act_dtype) -> int:
    return int(load().moe_grouped_ffn_wq_workspace_bytes(R, d, F, E, _DT[act_dtype]))


def moe_grouped_ffn_wq(x_perm, expert_offsets, E: int, d: int, F: int, bits: int, group_size: int,
                       w1_packed, s1, w2_packed, s2, b1=None, b2=None, y_dtype=None, y_perm=None,
                       workspace=None, max_rows_per_expert: int = 0, activation: str = "relu"):
    R = x_perm.shape[0]
    y_dtype = y_dtype or x_perm.dtype
    if y_perm is None:
        y_perm = torch.empty((R, d), dtype=y_dtype, device=x_perm.device)
    if workspace is None:
        workspace = torch.empty(moe_grouped_ffn_wq_workspace_bytes(R, d, F, E, x_perm.dtype),
                                dtype=torch.uint8, device=x_perm.device)
    rc = load().moe_grouped_ffn_wq(
        _ptr(x_perm, (torch.float16, torch.bfloat16), "x_perm"), _DT[x_perm.dtype],
        _ptr(expert_offsets, torch.int32, "expert_offsets"), R, E, max_rows_per_expert, d, F, bits, group_size,
        ACTIVATIONS[activation],
        _ptr(w1_packed, torch.uint8, "w1_packed"), _ptr(s1, torch.float16, "s1"), _ptr(b1, torch.float16, "b1"),
        _ptr(w2_packed, torch.uint8, "w2_packed"), _ptr(s2, torch.float16, "s2"), _ptr(b2, torch.float16, "b2"),
        _ptr(y_perm), _DT[y_perm.dtype], _ptr(workspace), workspace.numel(), _stream())
    _check(rc, "moe_grouped_ffn_wq")
    return y_perm


def moe_grouped_ffn_wq_noalloc(x_perm, expert_offsets, E: int, d: int, F: int, bits: int, group_size: int,
                               w1_packed, s1, w2_packed, s2, y_perm, b1=None, b2=None,
                               max_rows_per_expert: int = 0, activation: str = "relu"):
    """moe_grouped_ffn_wq without a workspace (scratch inside the library); y_perm is the caller's."""
    R = x_perm.shape[0]
    rc = load().moe_grouped_ffn_wq_noalloc(
        _ptr(x_perm, (torch.float16, torch.bfloat16), "x_perm"), _DT[x_perm.dtype],
        _ptr(expert_offsets, torch.int32, "expert_offsets"), R, E, max_rows_per_expert, d, F, bits, group_size,
        ACTIVATIONS[activation],
        _ptr(w1_packed, torch.uint8, "w1_packed"), _ptr(s1, torch.float16, "s1"), _ptr(b1, torch.float16, "b1"),
        _ptr(w2_packed, torch.uint8, "w2_packed"), _ptr(s2, torch.float16, "s2"), _ptr(b2, torch.float16, "b2"),
        _ptr(y_perm), _DT[y_perm.dtype], _stream())
    _check(rc, "moe_grouped_ffn_wq_noalloc")
    return y_perm


def moe_combine(y_perm, inv_perm, expert_scale, T: int, k: int, out_dtype=torch.float32, out=None,
                active_rows=None):
    """active_rows: a one-element int32 view (expert_offsets[E:E+1]) when rows may be pruned."""
    d = y_perm.shape[1]
    if out is None:
        out = torch.empty((T, d), dtype=out_dtype, device=y_perm.device)
    rc = load().moe_combine(_ptr(y_perm), _DT[y_perm.dtype], _ptr(inv_perm, torch.int32, "inv_perm"),
                            _ptr(expert_scale, torch.float32, "expert_scale"),
                            _ptr(active_rows, torch.int32, "active_rows"), T, k, d, _ptr(out),
                            _DT[out.dtype], _stream())
    _check(rc, "moe_combine")
    return out


def moe_pack_fp16_experts(w):
    """w fp32 [E,K,N] -> fp16 weights in the fragment layout (uint8, E*K*N*2 bytes)."""
    E, K, N = w.shape
    packed = torch.empty(E * K * N * 2, dtype=torch.uint8, device=w.device)
    rc = load().moe_pack_fp16_experts(_ptr(w, torch.float32, "w"), E, K, N, _ptr(packed), _stream())
    _check(rc, "moe_pack_fp16_experts")
    return packed


def moe_grouped_gemm_wq(x_perm, expert_offsets, E: int, K: int, N: int, bits: int, w_packed, scales=None,
                        native_convert: bool = False, y_dtype=None, y=None, max_rows_per_expert: int = 0):
    """One grouped GEMM of the decode-sized case (Table 1): y[r] = x_perm[r] @ deq(W[e])."""
    R = x_perm.shape[0]
    if y is None:
        y = torch.empty((R, N), dtype=y_dtype or x_perm.dtype, device=x_perm.device)
    rc = load().moe_grouped_gemm_wq(_ptr(x_perm, torch.float16, "x_perm"), _ptr(expert_offsets, torch.int32, "expert_offsets"),
                                    R, E, max_rows_per_expert, K, N, bits, int(native_convert),
                                    _ptr(w_packed, torch.uint8, "w_packed"), _ptr(scales, torch.float16, "scales"),
                                    _ptr(y), _DT[y.dtype], _stream())
    _check(rc, "moe_grouped_gemm_wq")
    return y


def moe_grouped_ffn_wq_routed_supported(R: int, E: int, max_rows_per_expert: int, d: int, F: int, bits: int,
                                        group_size: int, act_dtype) -> bool:
    return bool(load().moe_grouped_ffn_wq_routed_supported(R, E, max_rows_per_expert, d, F, bits, group_size,
                                                           _DT[act_dtype]))


def moe_grouped_ffn_wq_routed(x, perm_src, k: int, expert_offsets, E: int, d: int, F: int, bits: int, group_size: int,
                              w1_packed, s1, w2_packed, s2, b1=None, b2=None, expert_scale=None, out=None,
                              out_dtype=None, workspace=None, max_rows_per_expert: int = 0, activation: str = "relu"):
    """FFN with the gather (and, with expert_scale and k = 1, the combine) fused into the GEMMs."""
    R = perm_src.shape[0]
    T = x.shape[0]
    if out is None:
        out = torch.empty((T if expert_scale is not None else R, d), dtype=out_dtype or x.dtype, device=x.device)
    if workspace is None:
        workspace = torch.empty(moe_grouped_ffn_wq_workspace_bytes(R, d, F, E, x.dtype), dtype=torch.uint8, device=x.device)
    rc = load().moe_grouped_ffn_wq_routed(
        _ptr(x, torch.float16, "x"), _DT[x.dtype], _ptr(perm_src, torch.int32, "perm_src"), k,
        _ptr(expert_scale, torch.float32, "expert_scale"), _ptr(expert_offsets, torch.int32, "expert_offsets"), R, E,
        max_rows_per_expert, d, F, bits, group_size, ACTIVATIONS[activation], _ptr(w1_packed, torch.uint8, "w1_packed"),
        _ptr(s1, torch.float16, "s1"),
        _ptr(b1, torch.float16, "b1"), _ptr(w2_packed, torch.uint8, "w2_packed"), _ptr(s2, torch.float16, "s2"),
        _ptr(b2, torch.float16, "b2"), _ptr(out), _DT[out.dtype], _ptr(workspace), workspace.numel(), _stream())
    _check(rc, "moe_grouped_ffn_wq_routed")
    return out


def moe_grouped_ffn_wq_indexed_pays(R: int, E: int, max_rows_per_expert: int, d: int, F: int, bits: int, group_size: int, act_dtype) -> bool:
    """Whether fetching the rows through the routing index is the faster way for these sizes."""
    return bool(load().moe_grouped_ffn_wq_indexed_pays(R, E, max_rows_per_expert, d, F, bits, group_size, _DT[act_dtype]))


def moe_grouped_ffn_wq_unsorted_pays(T: int, k: int, E: int, d: int, F: int, bits: int, group_size: int, act_dtype) -> bool:
    """Whether the unsorted call is taken and the faster way for these sizes."""
    return bool(load().moe_grouped_ffn_wq_unsorted_pays(T, k, E, d, F, bits, group_size, _DT[act_dtype]))


def moe_grouped_ffn_wq_unsorted(x, expert_idx, E: int, d: int, F: int, bits: int, group_size: int, w1_packed, s1, w2_packed, s2,
                                b1=None, b2=None, expert_scale=None, out_dtype=None, workspace=None, activation: str = "relu"):
    """Index and FFN in row tiles in one call.  Returns (y_perm [R,d] or, with expert_scale, out [T,d], perm_src, inv_perm, expert_offsets)."""
    T, k = expert_idx.shape
    R = T * k
    dev = x.device
    out = torch.empty((T if expert_scale is not None else R, d), dtype=out_dtype or x.dtype, device=dev)
    perm_src = torch.empty(R, dtype=torch.int32, device=dev)
    inv_perm = torch.empty(R, dtype=torch.int32, device=dev)
    offsets = torch.empty(E + 1, dtype=torch.int32, device=dev)
    if workspace is None:
        workspace = torch.empty(moe_grouped_ffn_wq_workspace_bytes(R, d, F, E, x.dtype), dtype=torch.uint8, device=dev)
    rc = load().moe_grouped_ffn_wq_unsorted(
        _ptr(x, (torch.float16, torch.bfloat16), "x"), _DT[x.dtype], _ptr(expert_idx, torch.int32, "expert_idx"),
        _ptr(expert_scale, torch.float32, "expert_scale"), T, k, E, d, F, bits, group_size, ACTIVATIONS[activation],
        _ptr(w1_packed, torch.uint8, "w1_packed"), _ptr(s1, torch.float16, "s1"), _ptr(b1, torch.float16, "b1"),
        _ptr(w2_packed, torch.uint8, "w2_packed"), _ptr(s2, torch.float16, "s2"), _ptr(b2, torch.float16, "b2"), _ptr(out),
        _DT[out.dtype], _ptr(perm_src), _ptr(inv_perm), _ptr(offsets), _ptr(workspace), workspace.numel(), _stream())
    _check(rc, "moe_grouped_ffn_wq_unsorted")
    return out, perm_src, inv_perm, offsets


def moe_grouped_ffn_wq_gated_supported(T: int, k: int, E: int, d: int, F: int, bits: int, group_size: int, act_dtype) -> int:
    """0: not taken; 1: permute + FFN; 2: expert_scale may be given as well (combine fused in)."""
    return int(load().moe_grouped_ffn_wq_gated_supported(T, k, E, d, F, bits, group_size, _DT[act_dtype]))


def moe_grouped_ffn_wq_gated_pays(T: int, k: int, E: int, d: int, F: int, bits: int, group_size: int, act_dtype) -> bool:
    """Whether the gated call is also the faster way for these sizes."""
    return bool(load().moe_grouped_ffn_wq_gated_pays(T, k, E, d, F, bits, group_size, _DT[act_dtype]))


def moe_grouped_ffn_wq_gated(x, expert_idx, E: int, d: int, F: int, bits: int, group_size: int, w1_packed, s1, w2_packed,
                             s2, b1=None, b2=None, y_dtype=None, workspace=None, activation: str = "relu",
                             expert_scale=None):
    """Decode-sized batches: permute + FFN (+ combine when expert_scale is given) in one call.
    Returns (y_perm [R,d] or, with expert_scale, out [T,d] fp32, perm_src, inv_perm, expert_offsets)."""
    T, k = expert_idx.shape
    R = T * k
    dev = x.device
    if expert_scale is not None:
        y = torch.empty((T, d), dtype=torch.float32, device=dev)
    else:
        y = torch.empty((R, d), dtype=y_dtype or x.dtype, device=dev)
    perm_src = torch.empty(R, dtype=torch.int32, device=dev)
    inv_perm = torch.empty(R, dtype=torch.int32, device=dev)
    offsets = torch.empty(E + 1, dtype=torch.int32, device=dev)
    if workspace is None:
        workspace = torch.empty(moe_grouped_ffn_wq_workspace_bytes(R, d, F, E, x.dtype), dtype=torch.uint8, device=dev)
    rc = load().moe_grouped_ffn_wq_gated(
        _ptr(x, torch.float16, "x"), _DT[x.dtype], _ptr(expert_idx, torch.int32, "expert_idx"),
        _ptr(expert_scale, torch.float32, "expert_scale"), T, k, E, d, F, bits,
        group_size, ACTIVATIONS[activation], _ptr(w1_packed, torch.uint8, "w1_packed"), _ptr(s1, torch.float16, "s1"),
        _ptr(b1, torch.float16, "b1"), _ptr(w2_packed, torch.uint8, "w2_packed"), _ptr(s2, torch.float16, "s2"),
        _ptr(b2, torch.float16, "b2"), _ptr(y), _DT[y.dtype], _ptr(perm_src), _ptr(inv_perm), _ptr(offsets),
        _ptr(workspace), workspace.numel(), _stream())
    _check(rc, "moe_grouped_ffn_wq_gated")
    return y, perm_src, inv_perm, offsets


def moe_grouped_ffn_wq_sliced_workspace_bytes(T: int, k: int, E: int, d: int, F: int, bits: int, group_size: int, act_dtype) -> int:
    """0: not taken."""
    return int(load().moe_grouped_ffn_wq_sliced_workspace_bytes(T, k, E, d, F, bits, group_size, _DT[act_dtype]))


def moe_grouped_ffn_wq_sliced_pays(T: int, k: int, E: int, d: int, F: int, bits: int, group_size: int, act_dtype) -> bool:
    """Whether the sliced call is taken and the faster way for these sizes."""
    return bool(load().moe_grouped_ffn_wq_sliced_pays(T, k, E, d, F, bits, group_size, _DT[act_dtype]))


def moe_grouped_ffn_wq_sliced(x, expert_idx, expert_scale, E: int, d: int, F: int, bits: int, group_size: int, w1_packed, s1,
                              w2_packed, s2, b1=None, b2=None, out_dtype=torch.float32, workspace=None, activation: str = "relu"):
    """Few rows per expert: permute + FFN + combine in one call.  Returns (out [T,d], perm_src, inv_perm, expert_offsets)."""
    T, k = expert_idx.shape
    dev = x.device
    out = torch.empty((T, d), dtype=out_dtype, device=dev)
    perm_src = torch.empty(T * k, dtype=torch.int32, device=dev)
    inv_perm = torch.empty(T * k, dtype=torch.int32, device=dev)
    offsets = torch.empty(E + 1, dtype=torch.int32, device=dev)
    if workspace is None:
        workspace = torch.empty(max(256, moe_grouped_ffn_wq_sliced_workspace_bytes(T, k, E, d, F, bits, group_size, x.dtype)),
                                dtype=torch.uint8, device=dev)
    rc = load().moe_grouped_ffn_wq_sliced(
        _ptr(x, (torch.float16, torch.bfloat16), "x"), _DT[x.dtype], _ptr(expert_idx, torch.int32, "expert_idx"),
        _ptr(expert_scale, torch.float32, "expert_scale"), T, k, E, d, F, bits, group_size, ACTIVATIONS[activation],
        _ptr(w1_packed, torch.uint8, "w1_packed"), _ptr(s1, torch.float16, "s1"), _ptr(b1, torch.float16, "b1"),
        _ptr(w2_packed, torch.uint8, "w2_packed"), _ptr(s2, torch.float16, "s2"), _ptr(b2, torch.float16, "b2"), _ptr(out),
        _DT[out_dtype], _ptr(perm_src), _ptr(inv_perm), _ptr(offsets), _ptr(workspace), workspace.numel(), _stream())
    _check(rc, "moe_grouped_ffn_wq_sliced")
    return out, perm_src, inv_perm, offsets


# ---- microscaled 4-bit floating point (codes [.., R, K/2] and scales [.., ceil(K/128), R, 4], include/moe_wq.h) ----------------------

_FLOATS = (torch.float16, torch.bfloat16, torch.float32)


def moe_mx4_shapes(rows: int, K: int):
    """Shapes of the codes and the scales of `rows` rows of K values."""
    return (rows, K // 2), (-(-K // 128), rows, 4)


def _mx4_like(codes, scales, name):
    """(matrices or None, rows, K) of codes and scales that belong together."""
    cs = codes.shape
    if len(cs) == 2:
        (rows, half), matrices = cs, None
        want = (-(-half // 64), rows, 4)
    elif len(cs) == 3:
        matrices, rows, half = cs
        want = (matrices, -(-half // 64), rows, 4)
    else:
        half = 1
    if half % 32:
        raise MoeError("%s codes must be [R, K/2] or [E, N, K/2] with K %% 64 == 0, not %s" % (name, tuple(cs)))
    if scales.shape != want:
        raise MoeError("%s scales must be [.., ceil(K/128), rows, 4] beside codes %s, not %s" % (name, tuple(cs), tuple(scales.shape)))
    return matrices, rows, 2 * half


def moe_mx4_quantize_rows(x, out=None):
    """x [R, K] (rows may be strided) -> (codes uint8 [R, K/2], scales uint8 [ceil(K/128), R, 4])."""
    dtype = _DT.get(x.dtype)
    if dtype is None or x.dim() != 2 or not x.is_cuda:
        raise MoeError("x must be a [R, K] CUDA tensor of fp16, bf16 or fp32")
    (R, K), (stride, inner) = x.shape, x.stride()
    if inner != 1 and K > 1:
        raise MoeError("x must have contiguous rows")
    if R == 1:
        stride = K
    if out is None:
        dev = x.device
        codes, scales = torch.empty(R, K // 2, dtype=torch.uint8, device=dev), torch.empty(-(-K // 128), R, 4, dtype=torch.uint8, device=dev)
    else:
        codes, scales = out
        if _mx4_like(codes, scales, "out")[1:] != (R, K):
            raise MoeError("out does not fit x")
    rc = load().moe_mx4_quantize_rows(x.data_ptr(), dtype, R, K, stride, _ptr(codes, torch.uint8, "codes"),
                                      _ptr(scales, torch.uint8, "scales"), _stream())
    _check(rc, "moe_mx4_quantize_rows")
    return codes, scales


def moe_mx4_quantize_experts(w, out=None):
    """w fp32 [E, K, N] -> (codes uint8 [E, N, K/2], scales uint8 [E, ceil(K/128), N, 4])."""
    E, K, N = w.shape
    if out is None:
        cs, ss = moe_mx4_shapes(N, K)
        codes, scales = torch.empty((E,) + cs, dtype=torch.uint8, device=w.device), torch.empty((E,) + ss, dtype=torch.uint8, device=w.device)
    else:
        codes, scales = out
        if _mx4_like(codes, scales, "out") != (E, N, K):
            raise MoeError("out does not fit w")
    rc = load().moe_mx4_quantize_experts(_ptr(w, torch.float32, "w"), E, K, N, _ptr(codes, torch.uint8, "codes"), _ptr(scales, torch.uint8, "scales"), _stream())
    _check(rc, "moe_mx4_quantize_experts")
    return codes, scales


def moe_mx4_dequantize(codes, scales, dtype=torch.bfloat16, out=None):
    """The values that codes [.., R, K/2] and scales [.., ceil(K/128), R, 4] stand for, [.., R, K]."""
    matrices, rows, K = _mx4_like(codes, scales, "the")
    if out is None:
        out = (torch.empty(rows, K, dtype=dtype, device=codes.device) if matrices is None
               else torch.empty(matrices, rows, K, dtype=dtype, device=codes.device))
    elif tuple(out.shape) != tuple(codes.shape[:-1]) + (K,):
        raise MoeError("out must be %s" % (tuple(codes.shape[:-1]) + (K,),))
    rc = load().moe_mx4_dequantize(_ptr(codes, torch.uint8, "codes"), _ptr(scales, torch.uint8, "scales"), 1 if matrices is None else matrices, rows, K,
                                   _ptr(out, _FLOATS, "out"), _DT[out.dtype], _stream())
    _check(rc, "moe_mx4_dequantize")
    return out


def _mx4_experts(codes, scales, expert_offsets, bias, name):
    E, N, K = _mx4_like(codes, scales, name)
    if E is None or expert_offsets.numel() != E + 1 or (bias is not None and bias.shape != (E, N)):
        raise MoeError("%s must be [E, N, K/2] beside E + 1 offsets and a bias [E, N]" % name)
    return E, N, K


def moe_grouped_gemm_mx4(a_codes, a_scales, expert_offsets, w_codes, w_scales, bias=None, activation=None, perm_src=None, k: int = 1,
                         y_dtype=torch.float16, y=None, max_rows_per_expert: int = 0):
    """y[r] = act(a[perm_src[r] / k] @ W[e]^T + bias[e]) for the rows r of every expert e; rows behind the last expert's are not written."""
    E, N, K = _mx4_experts(w_codes, w_scales, expert_offsets, bias, "w")
    matrices, rows, Ka = _mx4_like(a_codes, a_scales, "a")
    if matrices is not None or Ka != K:
        raise MoeError("a must be [R, K/2] with the weights' K = %d" % K)
    R = rows if perm_src is None else perm_src.numel()
    if y is None:
        y = torch.empty(R, N, dtype=y_dtype, device=a_codes.device)
    elif y.shape != (R, N):
        raise MoeError("y must be %s" % ((R, N),))
    rc = load().moe_grouped_gemm_mx4(
        _ptr(a_codes, torch.uint8, "a_codes"), _ptr(a_scales, torch.uint8, "a_scales"), rows, _ptr(perm_src, torch.int32, "perm_src"), k,
        _ptr(expert_offsets, torch.int32, "expert_offsets"), R, E, max_rows_per_expert, K, N, _ptr(w_codes, torch.uint8, "w_codes"),
        _ptr(w_scales, torch.uint8, "w_scales"), _ptr(bias, torch.float16, "bias"), -1 if activation is None else ACTIVATIONS[activation],
        _ptr(y, _FLOATS, "y"), _DT[y.dtype], _stream())
    _check(rc, "moe_grouped_gemm_mx4")
    return y


def moe_grouped_ffn_mx4_workspace_bytes(T: int, R: int, d: int, F: int) -> int:
    return int(load().moe_grouped_ffn_mx4_workspace_bytes(T, R, d, F))


def moe_grouped_ffn_mx4(x, expert_offsets, w1_codes, w1_scales, w2_codes, w2_scales, b1=None, b2=None, perm_src=None, k: int = 1, y_dtype=None,
                        y_perm=None, activation: str = "relu", max_rows_per_expert: int = 0, workspace=None):
    """Expert FFN on 4-bit weights: x [T, d] -> y_perm [R, d], R = perm_src's length (T without one); rows behind the last expert's are not written."""
    T, d = x.shape
    E, F, K1 = _mx4_experts(w1_codes, w1_scales, expert_offsets, b1, "w1")
    E2, d2, K2 = _mx4_experts(w2_codes, w2_scales, expert_offsets, b2, "w2")
    if (E2, d2, K2, K1) != (E, d, F, d):
        raise MoeError("w1 must be [E, F, d/2] and w2 [E, d, F/2] with x's d = %d" % d)
    R = T if perm_src is None else perm_src.numel()
    if y_perm is None:
        y_perm = torch.empty(R, d, dtype=y_dtype or x.dtype, device=x.device)
    elif y_perm.shape != (R, d):
        raise MoeError("y_perm must be %s" % ((R, d),))
    lib = load()
    if workspace is None:
        workspace = torch.empty(lib.moe_grouped_ffn_mx4_workspace_bytes(T, R, d, F), dtype=torch.uint8, device=x.device)
    rc = lib.moe_grouped_ffn_mx4(
        _ptr(x, _FLOATS, "x"), _DT[x.dtype], T, _ptr(perm_src, torch.int32, "perm_src"), k, _ptr(expert_offsets, torch.int32, "expert_offsets"), R, E,
        max_rows_per_expert, d, F, ACTIVATIONS[activation], _ptr(w1_codes, torch.uint8, "w1_codes"), _ptr(w1_scales, torch.uint8, "w1_scales"),
        _ptr(b1, torch.float16, "b1"), _ptr(w2_codes, torch.uint8, "w2_codes"), _ptr(w2_scales, torch.uint8, "w2_scales"), _ptr(b2, torch.float16, "b2"),
        _ptr(y_perm, _FLOATS, "y_perm"), _DT[y_perm.dtype], _ptr(workspace, torch.uint8, "workspace"), workspace.numel(), _stream())
    _check(rc, "moe_grouped_ffn_mx4")
    return y_perm


# ---- the router's balance loss -------------------------------------------------------------------------------------------------------

def _check_balance(logits, expert_idx):
    z, i = logits.shape, expert_idx.shape
    if len(z) != 2 or len(i) != 2 or z[0] != i[0]:
        raise MoeError("logits must be [T, E] and expert_idx [T, k]")


def moe_balance_loss_workspace_bytes(T: int, E: int) -> int:
    return int(load().moe_balance_loss_workspace_bytes(T, E))


def moe_balance_loss(logits, expert_idx, coef: float = 0.01, renormalize: bool = True, workspace=None):
    """(loss [], counts int32 [E], prob_mean [E], expert_scale [T, k], weight [E]); weight is what moe_balance_loss_backward takes."""
    _check_balance(logits, expert_idx)
    (T, E), k, dev = logits.shape, expert_idx.shape[1], logits.device
    lib = load()
    # (tensors of their own, three allocations: views of one share a version counter, so that changing one in place would spoil the others for autograd)
    loss, prob_mean, weight = (torch.empty(shape, dtype=torch.float32, device=dev) for shape in ((), (E,), (E,)))
    counts = torch.empty(E, dtype=torch.int32, device=dev)
    scale = torch.empty(T, k, dtype=torch.float32, device=dev)
    if workspace is None:
        need = lib.moe_balance_loss_workspace_bytes(T, E)
        workspace = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    rc = lib.moe_balance_loss(_ptr(logits, _FLOATS, "logits"), _DT[logits.dtype], _ptr(expert_idx, torch.int32, "expert_idx"), T, E, k, int(renormalize),
                              coef, loss.data_ptr(), counts.data_ptr(), prob_mean.data_ptr(), scale.data_ptr(), weight.data_ptr(), _ptr(workspace, torch.uint8, "workspace"),
                              0 if workspace is None else workspace.numel(), _stream())
    _check(rc, "moe_balance_loss")
    return loss, counts, prob_mean, scale, weight


def moe_balance_loss_backward(logits, expert_idx, weight, dloss=None, dscale=None, renormalize: bool = True, out=None):
    """Gradient of moe_balance_loss's loss and expert_scale with respect to the logits, in their type."""
    _check_balance(logits, expert_idx)
    (T, E), k = logits.shape, expert_idx.shape[1]
    if weight.numel() != E or (dloss is not None and dloss.numel() != 1) or (dscale is not None and dscale.shape != (T, k)):
        raise MoeError("weight must be [E], dloss one number and dscale [T, k]")
    if out is None:
        out = torch.empty_like(logits)
    elif out.shape != logits.shape:
        raise MoeError("out must have the shape of logits")
    rc = load().moe_balance_loss_backward(_ptr(logits, _FLOATS, "logits"), _DT[logits.dtype], _ptr(expert_idx, torch.int32, "expert_idx"), T, E, k,
                                          int(renormalize), _ptr(weight, torch.float32, "weight"), _ptr(dloss, torch.float32, "dloss"),
                                          _ptr(dscale, torch.float32, "dscale"), _ptr(out, logits.dtype, "out"), _stream())
    _check(rc, "moe_balance_loss_backward")
    return out
