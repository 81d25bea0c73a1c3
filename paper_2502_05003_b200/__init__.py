"""B200 (sm_100a) implementation of the QuEST quantized-linear forward pass (arXiv 2502.05003,
Algorithm 1).  This module is a thin binding over the C ABI in ``include/quest.h``: it marshals
torch tensors (device memory, current stream) into pointers and sizes; every step of the path
runs in the CUDA library.  There is no CPU or PyTorch fallback.  The per-layer calls go through a
CPython binding (``csrc/quest_binding.cpp``) when their arguments are the plain case and through
ctypes otherwise, with the same outcome.
"""
from __future__ import annotations

import ctypes

import torch

from . import _lib
from ._lib import QuestError  # noqa: F401

F32, BF16 = 0, 1
_DT = {torch.float32: F32, torch.bfloat16: BF16}


def container_bits(bits: int) -> int:
    return 1 if bits == 1 else 2 if bits == 2 else 4 if bits <= 4 else 8


def _p(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype not in _DT:
        raise TypeError(f"unsupported dtype {t.dtype}: float32 or bfloat16")
    return _DT[t.dtype]


def _require_cuda(*ts):
    for t in ts:
        if t is not None and not t.is_cuda:
            raise ValueError("quest: tensors must live in CUDA device memory")


def _dense_operands(name: str, x: torch.Tensor, w: torch.Tensor):
    """x and w as the library reads them: rows one after the other, one dtype, one row length (w None: cached)."""
    if w is not None:
        if w.dim() != 2 or w.shape[1] != x.shape[1]:
            raise ValueError(f"{name}: x [M, K] and w [N, K]")
        if w.dtype != x.dtype:
            raise TypeError(f"{name}: x and w share one dtype")
        w = w.contiguous()
    return x.contiguous(), w


def _require_room(name: str, **tensors):
    """Every (tensor, bytes) is stored densely in CUDA memory and holds that many bytes (None: not given)."""
    for key, (t, nbytes) in tensors.items():
        if t is None:
            continue
        _require_cuda(t)
        if not t.is_contiguous() or t.numel() * t.element_size() < nbytes:
            raise ValueError(f"{name}: {key} must be contiguous and hold {nbytes} bytes")


def _result(done):
    """What the CPython binding returned for a call it made: the result, or the status of a call the library refused."""
    if done.__class__ is int:
        _lib.check(done)
    return done


def quest_alpha_star(bits: int) -> float:
    return float(_lib.load().quest_alpha_star(bits))


def quest_codes_bytes(rows: int, cols: int, bits: int) -> int:
    return int(_lib.load().quest_codes_bytes(rows, cols, bits))


def quest_workspace_bytes(M: int, N: int, K: int, bits_x: int, bits_w: int) -> int:
    return int(_lib.load().quest_workspace_bytes(M, N, K, bits_x, bits_w))


def quest_device_status() -> int:
    return int(_lib.load().quest_device_status(_stream()))


def quest_last_device_status() -> int:
    return int(_lib.load().quest_last_device_status(_stream()))


def quest_selftest_bounded_wait(limit_cycles: int = 2_000_000) -> torch.Tensor:
    """Makes a bounded wait of the kernels run out on purpose (harmless: one warp, a barrier nothing completes).
    Returns the 4-int device report; afterwards ``quest_device_status()`` is 12 once, then 0."""
    report = torch.full((4,), -1, dtype=torch.int32, device="cuda")
    _lib.check(_lib.load().quest_selftest_bounded_wait(limit_cycles, _p(report), _stream()))
    return report


STAGES = ("quant_x", "quant_w", "unpack", "gemm")


def quest_stage_timing(enable: bool) -> None:
    _lib.check(_lib.load().quest_stage_timing(1 if enable else 0))


def quest_stage_times(reset=False) -> dict:
    """Collects the events of the latest call (or, for calls captured into a CUDA graph, of the
    latest replay); returns {stage: (total_ms, count)}.  ``reset``: False/0 keep the totals,
    True/1 zero them, 2 also forget stages recorded inside a capture."""
    tot = (ctypes.c_double * len(STAGES))()
    cnt = (ctypes.c_longlong * len(STAGES))()
    _lib.check(_lib.load().quest_stage_times(tot, cnt, int(reset)))
    return {name: (float(tot[i]), int(cnt[i])) for i, name in enumerate(STAGES)}


def alloc_workspace(M: int, N: int, K: int, bits_x: int, bits_w: int, device=None) -> torch.Tensor:
    n = quest_workspace_bytes(M, N, K, bits_x, bits_w)
    if n == 0:
        raise ValueError("quest: invalid GEMM shape or bit-widths")
    return torch.empty(n, dtype=torch.uint8, device=device or torch.device("cuda"))


def quest_quantize(x: torch.Tensor, bits: int, had_block: int, trust_factor: float = 1.0,
                   codes: torch.Tensor = None, scales: torch.Tensor = None, mask: torch.Tensor = None,
                   want_mask: bool = True):
    """Rows of ``x`` [rows, cols] -> (codes uint8 [rows, cols*container/8], scales f32 [rows],
    mask uint8 [rows, cols/8] or None)."""
    done = _lib.binding().quantize(x, bits, had_block, trust_factor, codes, scales, mask, want_mask)
    if done is not None:
        return _result(done)
    _require_cuda(x, codes, scales, mask)
    if x.dim() != 2 or x.stride(1) != 1:
        raise ValueError("quest_quantize: x must be 2-D with unit inner stride")
    rows, cols = x.shape
    cb = container_bits(bits) if 1 <= bits <= 8 else 8
    if codes is None:
        codes = torch.empty((rows, cols * cb // 8), dtype=torch.uint8, device=x.device)
    if scales is None:
        scales = torch.empty(rows, dtype=torch.float32, device=x.device)
    if mask is None and want_mask:
        mask = torch.empty((rows, cols // 8), dtype=torch.uint8, device=x.device)
    st = _lib.load().quest_quantize(_p(x), _dtype_code(x), rows, cols, x.stride(0), bits, had_block,
                                    ctypes.c_float(trust_factor), _p(codes), _p(scales), _p(mask), _stream())
    _lib.check(st)
    return codes, scales, mask


def quest_trust_mask(x: torch.Tensor, bits: int, had_block: int, trust_factor: float = 1.0,
                     mask: torch.Tensor = None) -> torch.Tensor:
    _require_cuda(x, mask)
    if x.dim() != 2 or x.stride(1) != 1:
        raise ValueError("quest_trust_mask: x must be 2-D with unit inner stride")
    rows, cols = x.shape
    if mask is None:
        mask = torch.empty((rows, cols // 8), dtype=torch.uint8, device=x.device)
    st = _lib.load().quest_trust_mask(_p(x), _dtype_code(x), rows, cols, x.stride(0), bits, had_block,
                                      ctypes.c_float(trust_factor), _p(mask), _stream())
    _lib.check(st)
    return mask


def quest_lowbit_gemm(xq: torch.Tensor, sx: torch.Tensor, bits_x: int,
                      wq: torch.Tensor, sw: torch.Tensor, bits_w: int, K: int,
                      out_dtype=torch.bfloat16, y: torch.Tensor = None, want_acc: bool = False,
                      acc: torch.Tensor = None, workspace: torch.Tensor = None, want_y: bool = True):
    """Packed codes -> (y [M, N] or None, acc int32 [M, N] or None)."""
    done = _lib.binding().lowbit_gemm(xq, sx, bits_x, wq, sw, bits_w, K, out_dtype, y, want_acc, acc, workspace, want_y)
    if done is not None:
        return _result(done)
    _require_cuda(xq, sx, wq, sw, y, acc, workspace)
    M, N = xq.shape[0], wq.shape[0]
    if y is None and want_y:
        y = torch.empty((M, N), dtype=out_dtype, device=xq.device)
    if acc is None and want_acc:
        acc = torch.empty((M, N), dtype=torch.int32, device=xq.device)
    if workspace is None:
        workspace = alloc_workspace(M, N, K, bits_x, bits_w, xq.device)
    st = _lib.load().quest_lowbit_gemm(_p(xq), _p(sx), bits_x, _p(wq), _p(sw), bits_w, M, N, K,
                                       _p(y), _dtype_code(y) if y is not None else 0,
                                       y.stride(0) if y is not None else N, _p(acc),
                                       _p(workspace), workspace.numel(), _stream())
    _lib.check(st)
    return y, acc


STATIC_SCRATCH_BYTES = 4 << 20


def quest_lowbit_gemm_static(xq: torch.Tensor, sx: torch.Tensor, bits_x: int,
                             wq: torch.Tensor, sw: torch.Tensor, bits_w: int, K: int,
                             y: torch.Tensor = None, acc: torch.Tensor = None):
    """``quest_lowbit_gemm`` for callers that cannot allocate: the int8 operands go to a fixed
    array inside the library instead of a workspace tensor.  The caller passes every output
    (``y`` and/or ``acc``) preallocated, so neither this wrapper nor the library allocates.
    Raises ``QuestError`` (status 13) when (M + N) * K needs more than ``STATIC_SCRATCH_BYTES``.
    Calls share the one array per device: keep them on one stream."""
    _require_cuda(xq, sx, wq, sw, y, acc)
    if y is None and acc is None:
        raise ValueError("quest_lowbit_gemm_static: pass y and/or acc preallocated")
    M, N = xq.shape[0], wq.shape[0]
    st = _lib.load().quest_lowbit_gemm_static(_p(xq), _p(sx), bits_x, _p(wq), _p(sw), bits_w, M, N, K,
                                              _p(y), _dtype_code(y) if y is not None else 0,
                                              y.stride(0) if y is not None else N, _p(acc), _stream())
    _lib.check(st)
    return y, acc


def quest_linear_fwd(x: torch.Tensor, w: torch.Tensor, bits: int, had_block: int, trust_factor: float = 1.0,
                     out_dtype=None, y: torch.Tensor = None, saved: dict = None, w_cached: dict = None,
                     workspace: torch.Tensor = None, want_masks: bool = True) -> dict:
    """Algorithm 1: returns {"y", "xq", "sx", "mx", "wq", "sw", "mw"}.

    ``saved`` may carry preallocated output tensors under those keys; ``w_cached`` = {"wq", "sw"}
    from an earlier call skips the weight quantization (then ``w`` may be None).  With
    ``w_cached["operand_in_workspace"]`` true the call also skips unpacking ``wq``: ``workspace``
    must be the tensor an earlier call for the same w used, untouched since (M may differ).
    ``x`` or ``w`` with other strides than those of a dense tensor is copied first; tensors that the
    call writes to, and cached ones, must be dense.
    """
    done = _lib.binding().linear_fwd(x, w, bits, had_block, trust_factor, out_dtype, y, saved, w_cached, workspace,
                                      want_masks)
    if done is not None:
        return _result(done)
    _require_cuda(x, w, y, workspace)
    M, K = x.shape
    out = dict(saved or {})
    if w_cached is not None:
        out["wq"], out["sw"] = w_cached["wq"], w_cached["sw"]
        N = out["wq"].shape[0]
        x, _ = _dense_operands("quest_linear_fwd", x, None)
    else:
        N = w.shape[0]
        x, w = _dense_operands("quest_linear_fwd", x, w)
    cb = container_bits(bits) if 1 <= bits <= 8 else 8
    dev = x.device

    def need(key, shape, dtype):
        if out.get(key) is None:
            out[key] = torch.empty(shape, dtype=dtype, device=dev)

    need("xq", (M, K * cb // 8), torch.uint8)
    need("sx", (M,), torch.float32)
    if w_cached is None:
        need("wq", (N, K * cb // 8), torch.uint8)
        need("sw", (N,), torch.float32)
    if want_masks:
        need("mx", (M, K // 8), torch.uint8)
        if w_cached is None:
            need("mw", (N, K // 8), torch.uint8)
    out.setdefault("mx", None)
    out.setdefault("mw", None)
    if y is None:
        y = torch.empty((M, N), dtype=out_dtype or x.dtype, device=dev)
    if workspace is None:
        workspace = alloc_workspace(M, N, K, bits, bits, dev)
    if 1 <= bits <= 8:
        _require_room("quest_linear_fwd", y=(y, M * N * y.element_size()), xq=(out["xq"], M * (K * cb // 8)), sx=(out["sx"], 4 * M),
                      mx=(out["mx"], M * (K // 8)), wq=(out["wq"], N * (K * cb // 8)), sw=(out["sw"], 4 * N),
                      mw=(out["mw"] if w_cached is None else None, N * (K // 8)))
    st = _lib.load().quest_linear_fwd(
        _p(x), _p(w), _dtype_code(x), M, N, K, bits, had_block, ctypes.c_float(trust_factor),
        _p(y), _dtype_code(y), _p(out["xq"]), _p(out["sx"]), _p(out["mx"]),
        _p(out["wq"]), _p(out["sw"]), _p(out["mw"]),
        0 if w_cached is None else (2 if w_cached.get("operand_in_workspace") else 1),
        _p(workspace), workspace.numel(), _stream())
    _lib.check(st)
    out["y"] = y
    return out


def quest_linear_fwd_quantize(x: torch.Tensor, w: torch.Tensor, bits: int, had_block: int, trust_factor: float,
                              saved: dict, workspace: torch.Tensor) -> None:
    """First half of ``quest_linear_fwd``: codes, scales, masks into ``saved`` (preallocated, keys xq, sx, mx, wq,
    sw, mw) and the tensor-core operands into ``workspace``."""
    _require_cuda(x, w, workspace)
    M, K = x.shape
    N = w.shape[0]
    x, w = _dense_operands("quest_linear_fwd_quantize", x, w)
    st = _lib.load().quest_linear_fwd_quantize(
        _p(x), _p(w), _dtype_code(x), M, N, K, bits, had_block, ctypes.c_float(trust_factor),
        _p(saved["xq"]), _p(saved["sx"]), _p(saved.get("mx")), _p(saved["wq"]), _p(saved["sw"]), _p(saved.get("mw")), 0,
        _p(workspace), workspace.numel(), _stream())
    _lib.check(st)


def quest_linear_fwd_contract(saved: dict, M: int, N: int, K: int, bits: int, y: torch.Tensor, workspace: torch.Tensor) -> None:
    """Second half of ``quest_linear_fwd``: the contraction of the operands that ``quest_linear_fwd_quantize`` left
    in ``workspace``, scaled by ``saved["sx"]`` and ``saved["sw"]``, into ``y``."""
    _require_cuda(y, workspace)
    st = _lib.load().quest_linear_fwd_contract(_p(saved["sx"]), _p(saved["sw"]), M, N, K, bits, _p(y), _dtype_code(y),
                                               _p(workspace), workspace.numel(), _stream())
    _lib.check(st)


def quest_bwd_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(_lib.load().quest_bwd_workspace_bytes(M, N, K))


def quest_linear_bwd(dy: torch.Tensor, fwd: dict, bits: int, had_block: int, K: int, out_dtype=torch.float32,
                     dx: torch.Tensor = None, dw: torch.Tensor = None, want_dx: bool = True, want_dw: bool = True,
                     workspace: torch.Tensor = None) -> dict:
    """Algorithm 2 from the forward call's saved tensors (``fwd`` holds xq, sx, mx, wq, sw, mw).
    ``dy`` [M, N] bfloat16.  Returns {"dx": [M, K] or None, "dw": [N, K] or None}."""
    done = _lib.binding().linear_bwd(dy, fwd, bits, had_block, K, out_dtype, dx, dw, want_dx, want_dw, workspace)
    if done is not None:
        return _result(done)
    _require_cuda(dy, dx, dw, workspace, *[fwd[k] for k in ("xq", "sx", "mx", "wq", "sw", "mw")])
    if dy.dtype != torch.bfloat16 or not dy.is_contiguous():
        raise ValueError("quest_linear_bwd: dy must be a contiguous bfloat16 tensor")
    M, N = dy.shape
    if dx is None and want_dx:
        dx = torch.empty((M, K), dtype=out_dtype, device=dy.device)
    if dw is None and want_dw:
        dw = torch.empty((N, K), dtype=out_dtype, device=dy.device)
    if workspace is None:
        n = quest_bwd_workspace_bytes(M, N, K)
        if n == 0:
            raise ValueError("quest_linear_bwd: unsupported shape (M, N multiples of 8; K a multiple of 32, <= 16384)")
        workspace = torch.empty(n, dtype=torch.uint8, device=dy.device)
    out_t = dx if dx is not None else dw
    st = _lib.load().quest_linear_bwd(_p(dy), M, N, K, bits, had_block, _p(fwd["xq"]), _p(fwd["sx"]), _p(fwd["mx"]),
                                      _p(fwd["wq"]), _p(fwd["sw"]), _p(fwd["mw"]), _p(dx), _p(dw),
                                      _dtype_code(out_t) if out_t is not None else 0,
                                      _p(workspace), workspace.numel(), _stream())
    _lib.check(st)
    return {"dx": dx, "dw": dw}


# ---- MLP block: gate / up / SwiGLU / down, every linear layer Algorithm 1 -------------------------

class _MlpSaved(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("xq", "sx", "mx", "wgq", "swg", "mwg", "wuq", "swu", "mwu",
                                               "hq", "sh", "mh", "wdq", "swd", "mwd")]


def quest_mlp_workspace_bytes(T: int, H: int, I: int) -> int:
    return int(_lib.load().quest_mlp_workspace_bytes(T, H, I))


def mlp_buffers(T: int, H: int, I: int, bits: int, device=None, out_dtype=torch.bfloat16, want_masks: bool = True) -> dict:
    """Every output of ``quest_mlp_fwd`` and its workspace, allocated once (the call itself allocates nothing)."""
    dev = device or torch.device("cuda")
    cb = container_bits(bits)
    n = quest_mlp_workspace_bytes(T, H, I)
    if n == 0:
        raise ValueError("quest_mlp_fwd: unsupported shape (H, I multiples of 32, at most 16384)")
    u8 = lambda *s: torch.empty(s, dtype=torch.uint8, device=dev)
    f32 = lambda *s: torch.empty(s, dtype=torch.float32, device=dev)
    b = {"h": torch.empty((T, I), dtype=torch.bfloat16, device=dev), "y": torch.empty((T, H), dtype=out_dtype, device=dev),
         "xq": u8(T, H * cb // 8), "sx": f32(T), "wgq": u8(I, H * cb // 8), "swg": f32(I), "wuq": u8(I, H * cb // 8),
         "swu": f32(I), "hq": u8(T, I * cb // 8), "sh": f32(T), "wdq": u8(H, I * cb // 8), "swd": f32(H),
         "workspace": u8(n), "launches": 4}
    for k, shape in (("mx", (T, H // 8)), ("mwg", (I, H // 8)), ("mwu", (I, H // 8)), ("mh", (T, I // 8)), ("mwd", (H, I // 8))):
        b[k] = u8(*shape) if want_masks else None
    return b


def quest_mlp_fwd(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, bits: int,
                  had_block: int, trust_factor: float = 1.0, buffers: dict = None, out_dtype=torch.bfloat16) -> dict:
    """y = down(silu(gate(x)) * up(x)) with QuEST linear layers.  Returns the ``buffers`` dict: "y" [T, H],
    "h" [T, I] bfloat16 and the codes / scales / masks of x, w_gate, w_up, h, w_down."""
    done = _lib.binding().mlp_fwd(x, w_gate, w_up, w_down, bits, had_block, trust_factor, buffers)
    if done is not None:
        return _result(done)
    _require_cuda(x, w_gate, w_up, w_down)
    T, H = x.shape
    I = w_gate.shape[0]
    if w_up.shape != (I, H) or w_down.shape != (H, I) or not all(t.is_contiguous() for t in (x, w_gate, w_up, w_down)):
        raise ValueError("quest_mlp_fwd: x [T, H], w_gate / w_up [I, H], w_down [H, I], all contiguous")
    if not (x.dtype == w_gate.dtype == w_up.dtype == w_down.dtype):
        raise TypeError("quest_mlp_fwd: x and the weights share one dtype")
    b = buffers if buffers is not None else mlp_buffers(T, H, I, bits, x.device, out_dtype)
    sv = _MlpSaved(*[(b[n].data_ptr() if b.get(n) is not None else None) for n, _ in _MlpSaved._fields_])
    st = _lib.load().quest_mlp_fwd(_p(x), _p(w_gate), _p(w_up), _p(w_down), _dtype_code(x), T, H, I, bits, had_block,
                                   ctypes.c_float(trust_factor), _p(b["h"]), _p(b["y"]), _dtype_code(b["y"]),
                                   ctypes.byref(sv), _p(b["workspace"]), b["workspace"].numel(), _stream())
    _lib.check(st)
    return b


# ---- weight-only variant (Section 4.5): b-bit weights, bfloat16 activations -----------------------

def quest_weight_only_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(_lib.load().quest_weight_only_workspace_bytes(M, N, K))


def quest_linear_fwd_weight_only(x: torch.Tensor, w: torch.Tensor, bits_w: int, had_block: int,
                                 trust_factor: float = 1.0, out_dtype=torch.bfloat16, out: dict = None,
                                 workspace: torch.Tensor = None) -> dict:
    """y = HT(x) (kept in bfloat16) times the quantized w.  Returns {"y", "xh", "wq", "sw", "mw"};
    ``out`` may hold preallocated tensors under those keys."""
    done = _lib.binding().linear_fwd_weight_only(x, w, bits_w, had_block, trust_factor, out_dtype, out, workspace)
    if done is not None:
        return _result(done)
    _require_cuda(x, w, workspace)
    if x.dim() != 2 or w.dim() != 2 or x.stride(1) != 1 or w.stride(1) != 1 or x.shape[1] != w.shape[1]:
        raise ValueError("quest_linear_fwd_weight_only: x [M, K] and w [N, K] with unit inner stride")
    M, K = x.shape
    N = w.shape[0]
    out = dict(out) if out else {}
    cb = container_bits(bits_w)

    def need(key, shape, dtype):
        if out.get(key) is None:
            out[key] = torch.empty(shape, dtype=dtype, device=x.device)
        return out[key]

    y = need("y", (M, N), out_dtype)
    xh = need("xh", (M, K), torch.bfloat16)
    wq = need("wq", (N, K * cb // 8), torch.uint8)
    sw = need("sw", (N,), torch.float32)
    mw = need("mw", (N, K // 8), torch.uint8)
    _require_cuda(y, xh, wq, sw, mw)
    if workspace is None:
        n = quest_weight_only_workspace_bytes(M, N, K)
        if n == 0:
            raise ValueError("quest_linear_fwd_weight_only: unsupported shape (K a multiple of 32, 32 <= K <= 16384)")
        workspace = torch.empty(n, dtype=torch.uint8, device=x.device)
    st = _lib.load().quest_linear_fwd_weight_only(
        _p(x), _dtype_code(x), x.stride(0), _p(w), _dtype_code(w), w.stride(0), M, N, K, bits_w, had_block,
        ctypes.c_float(trust_factor), _p(y), _dtype_code(y), y.stride(0), _p(xh), _p(wq), _p(sw), _p(mw),
        _p(workspace), workspace.numel(), _stream())
    _lib.check(st)
    return out


# ---- FP4 (E2M1) grid variant: same calls with the FP4 rounding grid of Section 4.4 ---------------

def quest_alpha_star_fp4() -> float:
    return float(_lib.load().quest_alpha_star_fp4())


def quest_quantize_fp4(x: torch.Tensor, had_block: int, trust_factor: float = 1.0):
    """Rows of ``x`` -> (E2M1 codes uint8 [rows, cols/2], scales f32 [rows], mask uint8 [rows, cols/8])."""
    _require_cuda(x)
    if x.dim() != 2 or x.stride(1) != 1:
        raise ValueError("quest_quantize_fp4: x must be 2-D with unit inner stride")
    rows, cols = x.shape
    codes = torch.empty((rows, cols // 2), dtype=torch.uint8, device=x.device)
    scales = torch.empty(rows, dtype=torch.float32, device=x.device)
    mask = torch.empty((rows, cols // 8), dtype=torch.uint8, device=x.device)
    _lib.check(_lib.load().quest_quantize_fp4(_p(x), _dtype_code(x), rows, cols, x.stride(0), had_block,
                                              ctypes.c_float(trust_factor), _p(codes), _p(scales), _p(mask), _stream()))
    return codes, scales, mask


def quest_lowbit_gemm_fp4(xq, sx, wq, sw, K: int, out_dtype=torch.bfloat16, want_acc: bool = False, workspace=None):
    """E2M1 codes -> (y [M, N], acc4 int32 [M, N] or None); acc4 is four times the value product."""
    _require_cuda(xq, sx, wq, sw, workspace)
    M, N = xq.shape[0], wq.shape[0]
    y = torch.empty((M, N), dtype=out_dtype, device=xq.device)
    acc = torch.empty((M, N), dtype=torch.int32, device=xq.device) if want_acc else None
    # the packed codes are the tensor-core operands: the call needs no scratch (the argument is kept in the ABI)
    _lib.check(_lib.load().quest_lowbit_gemm_fp4(_p(xq), _p(sx), _p(wq), _p(sw), M, N, K, _p(y), _dtype_code(y),
                                                 y.stride(0), _p(acc), _p(workspace),
                                                 workspace.numel() if workspace is not None else 0, _stream()))
    return y, acc


def quest_linear_fwd_fp4(x: torch.Tensor, w: torch.Tensor, had_block: int, trust_factor: float = 1.0,
                         out_dtype=None, w_cached: dict = None, workspace: torch.Tensor = None) -> dict:
    """Algorithm 1 with the FP4 grid: returns {"y", "xq", "sx", "mx", "wq", "sw", "mw"}."""
    done = _lib.binding().linear_fwd_fp4(x, w, had_block, trust_factor, out_dtype, w_cached, workspace)
    if done is not None:
        return _result(done)
    _require_cuda(x, w, workspace)
    M, K = x.shape
    dev = x.device
    out = {}
    if w_cached is not None:
        out["wq"], out["sw"], out["mw"] = w_cached["wq"], w_cached["sw"], None
        N = out["wq"].shape[0]
        x, _ = _dense_operands("quest_linear_fwd_fp4", x, None)
        _require_room("quest_linear_fwd_fp4", wq=(out["wq"], N * (K // 2)), sw=(out["sw"], 4 * N))
    else:
        N = w.shape[0]
        x, w = _dense_operands("quest_linear_fwd_fp4", x, w)
        out["wq"] = torch.empty((N, K // 2), dtype=torch.uint8, device=dev)
        out["sw"] = torch.empty(N, dtype=torch.float32, device=dev)
        out["mw"] = torch.empty((N, K // 8), dtype=torch.uint8, device=dev)
    out["xq"] = torch.empty((M, K // 2), dtype=torch.uint8, device=dev)
    out["sx"] = torch.empty(M, dtype=torch.float32, device=dev)
    out["mx"] = torch.empty((M, K // 8), dtype=torch.uint8, device=dev)
    y = torch.empty((M, N), dtype=out_dtype or x.dtype, device=dev)
    _lib.check(_lib.load().quest_linear_fwd_fp4(
        _p(x), _p(w), _dtype_code(x), M, N, K, had_block, ctypes.c_float(trust_factor), _p(y), _dtype_code(y),
        _p(out["xq"]), _p(out["sx"]), _p(out["mx"]), _p(out["wq"]), _p(out["sw"]), _p(out["mw"]),
        1 if w_cached is not None else 0, _p(workspace), workspace.numel() if workspace is not None else 0, _stream()))
    out["y"] = y
    return out


# ---- microscaled (MX) layer: a power-of-two scale for every 32 elements; weights in 4 bits, activations in 4 or 8 -------

_MX_BLOCK = 32


def quest_mx_scales_bytes(rows: int, cols: int) -> int:
    """Bytes of the scales of an MX tensor (0 for a shape that the calls do not take)."""
    return int(_lib.load().quest_mx_scales_bytes(rows, cols))


def mx_scales_tiled(scales: torch.Tensor) -> torch.Tensor:
    """Scale bytes as checkpoints hold them, [rows, cols / 32], in the order that the calls take."""
    rows, blocks = scales.shape
    room = torch.zeros((-(-rows // 128) * 128, -(-blocks // 4) * 4), dtype=torch.uint8, device=scales.device)
    room[:rows, :blocks] = scales
    return room.reshape(-1, 4, 32, room.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).reshape(-1).contiguous()


def mx_scales_rows(scales: torch.Tensor, rows: int, cols: int) -> torch.Tensor:
    """The inverse of ``mx_scales_tiled``: [rows, cols / 32]."""
    tiles = -(-cols // 128)
    n = -(-rows // 128) * tiles * 512
    t = scales.reshape(-1)[:n].reshape(-1, tiles, 32, 4, 4).permute(0, 3, 2, 1, 4)
    return t.reshape(t.shape[0] * 128, tiles * 4)[:rows, :cols // _MX_BLOCK].contiguous()


def _beside(name: str, x: torch.Tensor, **tensors):
    """x and every tensor that is given are in the memory of one CUDA device."""
    _require_cuda(x, *tensors.values())
    for key, t in tensors.items():
        if t is not None and t.device != x.device:
            raise ValueError(f"{name}: {key} is on another device")


def _rows_of(name: str, key: str, t: torch.Tensor, shape=None):
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1) or (t.shape[0] > 1 and t.stride(0) < t.shape[1]):
        raise ValueError(f"{name}: {key} must be 2-D with unit inner stride")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: {key} must have the shape {tuple(shape)}")
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def _kept(name: str, out: dict, key: str, shape, dtype, device):
    """The tensor under ``key``, which must have that type and room for the shape, or a new one."""
    t = out.get(key)
    if t is None:
        t = out[key] = torch.empty(shape, dtype=dtype, device=device)
        return t
    n = 1
    for v in shape:
        n *= v
    if t.device != device or t.dtype != dtype or not t.is_contiguous() or t.numel() < n:
        raise ValueError(f"{name}: {key} must be a contiguous {dtype} tensor on {device} with {n} elements")
    return t


def _workspace_bytes_of(name: str, t) -> int:
    if t is None:
        return 0
    if not t.is_contiguous():
        raise ValueError(f"{name}: workspace must be contiguous")
    return t.numel() * t.element_size()


def _mx_codes_of(name: str, key: str, t: torch.Tensor, cols: int, bits: int):
    if t.dtype != torch.uint8 or t.dim() != 2 or not t.is_contiguous() or t.shape[1] * 8 != cols * bits:
        raise ValueError(f"{name}: {key} must be a contiguous uint8 tensor [rows, {cols * bits // 8}]")


def _mx_scales_of(name: str, key: str, t: torch.Tensor, rows: int, cols: int):
    if t.dtype != torch.uint8 or not t.is_contiguous() or t.numel() < quest_mx_scales_bytes(rows, cols):
        raise ValueError(f"{name}: {key} must be a contiguous uint8 tensor of {quest_mx_scales_bytes(rows, cols)} bytes")


def _product_out(name: str, y, M: int, N: int, out_dtype, device):
    if y is None:
        return torch.empty((M, N), dtype=out_dtype, device=device), max(N, 1)
    return y, _rows_of(name, "y", y, (M, N))


def _mx_check(name: str, bits: int):
    if bits not in (4, 8):
        raise ValueError(f"{name}: 4 or 8 bits")


def quest_quantize_mx(x: torch.Tensor, bits: int, had_block: int = 1, codes: torch.Tensor = None, scales: torch.Tensor = None):
    """Rows of ``x`` [rows, cols] -> (codes uint8 [rows, cols * bits / 8], scales uint8 [quest_mx_scales_bytes]).  ``bits``: 4
    (E2M1) or 8 (E4M3, ``codes.view(torch.float8_e4m3fn)``); ``had_block``: 1, or 32 for rotated blocks."""
    done = _lib.binding().quantize_mx(x, bits, had_block, codes, scales)
    if done is not None:
        return _result(done)
    name = "quest_quantize_mx"
    _beside(name, x, codes=codes, scales=scales)
    _mx_check(name, bits)
    ld, (rows, cols) = _rows_of(name, "x", x), x.shape
    out = {"codes": codes, "scales": scales}
    codes = _kept(name, out, "codes", (rows, cols * bits // 8), torch.uint8, x.device)
    scales = _kept(name, out, "scales", (quest_mx_scales_bytes(rows, cols),), torch.uint8, x.device)
    with torch.cuda.device(x.device):
        _lib.check(_lib.load().quest_quantize_mx(_p(x), _dtype_code(x), rows, cols, ld, bits, had_block, _p(codes), _p(scales), _stream()))
    return codes, scales


def quest_dequantize_mx(codes: torch.Tensor, scales: torch.Tensor, bits: int, out_dtype=torch.bfloat16, out: torch.Tensor = None):
    """Values [rows, cols] of an MX tensor, exact in binary32 and (down to 2^-133) in bfloat16; rotated where x was rotated."""
    done = _lib.binding().dequantize_mx(codes, scales, bits, out_dtype, out)
    if done is not None:
        return _result(done)
    name = "quest_dequantize_mx"
    _beside(name, codes, scales=scales, out=out)
    _mx_check(name, bits)
    if codes.dim() != 2:
        raise ValueError(f"{name}: codes must be 2-D")
    rows, cols = codes.shape[0], codes.shape[1] * 8 // bits
    _mx_codes_of(name, "codes", codes, cols, bits)
    _mx_scales_of(name, "scales", scales, rows, cols)
    out = _kept(name, {"out": out}, "out", (rows, cols), out_dtype if out is None else out.dtype, codes.device)
    with torch.cuda.device(codes.device):
        _lib.check(_lib.load().quest_dequantize_mx(_p(codes), _p(scales), rows, cols, bits, _p(out), _dtype_code(out), _stream()))
    return out


def quest_gemm_mx(xq: torch.Tensor, sx: torch.Tensor, bits_x: int, wq: torch.Tensor, sw: torch.Tensor, K: int,
                  out_dtype=torch.bfloat16, y: torch.Tensor = None) -> torch.Tensor:
    """y [M, N] = x w^T of two MX tensors: x in 4 or 8 bits, w in 4.  K a multiple of 32, of 128 where x has 8 bits."""
    done = _lib.binding().gemm_mx(xq, sx, bits_x, wq, sw, K, out_dtype, y)
    if done is not None:
        return _result(done)
    name = "quest_gemm_mx"
    _beside(name, xq, sx=sx, wq=wq, sw=sw, y=y)
    _mx_check(name, bits_x)
    _mx_codes_of(name, "xq", xq, K, bits_x)
    _mx_codes_of(name, "wq", wq, K, 4)
    M, N = xq.shape[0], wq.shape[0]
    _mx_scales_of(name, "sx", sx, M, K)
    _mx_scales_of(name, "sw", sw, N, K)
    with torch.cuda.device(xq.device):
        y, ldy = _product_out(name, y, M, N, out_dtype, xq.device)
        _lib.check(_lib.load().quest_gemm_mx(_p(xq), _p(sx), bits_x, _p(wq), _p(sw), M, N, K, _p(y), _dtype_code(y), ldy, _stream()))
    return y


def quest_mx_codes_optional(M: int, N: int, K: int) -> bool:
    """Whether ``quest_linear_fwd_mx`` can quantize x inside the product: M up to 8, M K up to 4096, N up to 7104."""
    return bool(_lib.load().quest_mx_codes_optional(M, N, K))


def quest_linear_fwd_mx(x: torch.Tensor, w: torch.Tensor, bits_x: int = 8, had_block: int = 1, out_dtype=None,
                        y: torch.Tensor = None, saved: dict = None, w_cached: dict = None, want_codes: bool = True) -> dict:
    """The microscaled layer, y = x w^T with x in ``bits_x`` bits and w in 4: returns {"y", "xq", "sx", "wq", "sw"}.

    ``saved`` may carry preallocated tensors for the codes and scales; ``w_cached`` = {"wq", "sw"} holds weights that are quantized
    already (then ``w`` may be None).  With ``want_codes`` false up to 8 rows of x (where ``quest_mx_codes_optional(M, N, K)``) are quantized
    inside the product and their codes are not stored (None); more rows need the room all the same.  ``x`` or ``w`` whose rows do not start on
    16-byte boundaries, or with another inner stride, is copied first."""
    done = _lib.binding().linear_fwd_mx(x, w, bits_x, had_block, out_dtype, y, saved, w_cached, want_codes)
    if done is not None:
        return _result(done)
    name = "quest_linear_fwd_mx"
    out = dict(saved or {})
    if w_cached is not None:
        out["wq"], out["sw"], w = w_cached["wq"], w_cached["sw"], None
    _beside(name, x, w=w, y=y, **{k: out.get(k) for k in ("xq", "sx", "wq", "sw")})
    _mx_check(name, bits_x)

    def rows(key, t):
        if t.dim() != 2:
            raise ValueError(f"{name}: {key} must be 2-D")
        if t.stride(1) != 1 or t.data_ptr() % 16 or (t.shape[0] > 1 and (t.stride(0) < t.shape[1] or t.stride(0) * t.element_size() % 16)):
            t = t.contiguous()
        if t.data_ptr() % 16:
            t = t.clone()
        return t, max(t.stride(0), t.shape[1])

    x, ldx = rows("x", x)
    M, K = x.shape
    dev = x.device
    with torch.cuda.device(dev):
        if w_cached is None:
            w, ldw = rows("w", w)
            N = w.shape[0]
            if w.shape[1] != K:
                raise ValueError(f"{name}: x [M, K] and w [N, K]")
            wdt = _dtype_code(w)
        else:
            _mx_codes_of(name, "wq", out["wq"], K, 4)
            N, ldw, wdt = out["wq"].shape[0], K, BF16
            _mx_scales_of(name, "sw", out["sw"], N, K)
        _kept(name, out, "wq", (N, K // 2), torch.uint8, dev)
        _kept(name, out, "sw", (quest_mx_scales_bytes(N, K),), torch.uint8, dev)
        if want_codes or not quest_mx_codes_optional(M, N, K):
            _kept(name, out, "xq", (M, K * bits_x // 8), torch.uint8, dev)
            _kept(name, out, "sx", (quest_mx_scales_bytes(M, K),), torch.uint8, dev)
        else:
            out["xq"] = out["sx"] = None
        y, ldy = _product_out(name, y, M, N, out_dtype or x.dtype, dev)
        _lib.check(_lib.load().quest_linear_fwd_mx(
            _p(x), _dtype_code(x), ldx, _p(w), wdt, ldw, M, N, K, bits_x, had_block, _p(y), _dtype_code(y), ldy,
            _p(out["xq"]), _p(out["sx"]), _p(out["wq"]), _p(out["sw"]), 0 if w_cached is None else 1, _stream()))
    out["y"] = y
    return out


def quest_bwd_mx_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(_lib.load().quest_bwd_mx_workspace_bytes(M, N, K))


def quest_linear_bwd_mx(dy: torch.Tensor, fwd: dict, bits_x: int, had_block: int, K: int, out_dtype=torch.float32,
                        dx: torch.Tensor = None, dw: torch.Tensor = None, want_dx: bool = True, want_dw: bool = True,
                        workspace: torch.Tensor = None) -> dict:
    """Gradients of ``quest_linear_fwd_mx`` straight through the rounding, from what it returned (xq, sx for dw; wq, sw for
    dx).  ``dy`` [M, N] bfloat16, dense.  Returns {"dx": [M, K] or None, "dw": [N, K] or None}; both have one type."""
    done = _lib.binding().linear_bwd_mx(dy, fwd, bits_x, had_block, K, out_dtype, dx, dw, want_dx, want_dw, workspace)
    if done is not None:
        return _result(done)
    name = "quest_linear_bwd_mx"
    want_dx, want_dw = want_dx or dx is not None, want_dw or dw is not None
    used = (["xq", "sx"] if want_dw else []) + (["wq", "sw"] if want_dx else [])
    _beside(name, dy, dx=dx, dw=dw, workspace=workspace, **{k: fwd.get(k) for k in used})
    _mx_check(name, bits_x)
    if dy.dtype != torch.bfloat16 or dy.dim() != 2 or not dy.is_contiguous():
        raise ValueError(f"{name}: dy must be a contiguous bfloat16 matrix")
    M, N = dy.shape
    n = quest_bwd_mx_workspace_bytes(M, N, K)
    if n == 0:
        raise ValueError(f"{name}: unsupported shape (M, N multiples of 8; K a multiple of 32, <= 16384)")
    for key in used:
        t, rows = fwd.get(key), M if key in ("xq", "sx") else N
        if t is None:
            raise ValueError(f"{name}: {key} of the forward call is missing")
        if key in ("xq", "wq"):
            _mx_codes_of(name, key, t, K, bits_x if key == "xq" else 4)
            if t.shape[0] != rows:
                raise ValueError(f"{name}: {key} must have {rows} rows")
        else:
            _mx_scales_of(name, key, t, rows, K)
    out = {"dx": dx, "dw": dw}
    given = dx if dx is not None else dw
    dt = out_dtype if given is None else given.dtype
    with torch.cuda.device(dy.device):
        if want_dx:
            _kept(name, out, "dx", (M, K), dt, dy.device)
        if want_dw:
            _kept(name, out, "dw", (N, K), dt, dy.device)
        if workspace is None:
            workspace = torch.empty(n, dtype=torch.uint8, device=dy.device)
        some = out["dx"] if out["dx"] is not None else out["dw"]
        _lib.check(_lib.load().quest_linear_bwd_mx(
            _p(dy), M, N, K, bits_x, had_block, *[_p(fwd[k]) if k in used else None for k in ("xq", "sx", "wq", "sw")],
            _p(out["dx"]), _p(out["dw"]), _dtype_code(some) if some is not None else F32, _p(workspace),
            _workspace_bytes_of(name, workspace), _stream()))
    return out


# ---- root-mean-square norm in front of a layer -------------------------------------------------------------------------

def quest_rmsnorm_fwd(x: torch.Tensor, weight: torch.Tensor, eps: float = 1e-5, residual: torch.Tensor = None, out_dtype=None,
                      mx_bits: int = None, had_block: int = 1, out: dict = None, want_rstd: bool = True) -> dict:
    """h = x + residual, y = h (mean(h^2) + eps)^(-1/2) weight for every row.  Returns {"h" (None without a residual),
    "rstd" [rows] or None, and "y" or, with ``mx_bits`` 4 or 8, "yq", "sy": the codes and scales that ``quest_gemm_mx``
    takes}.  ``out`` may hold preallocated tensors under those keys; "h" or "y" may be ``x`` or ``residual`` itself."""
    done = _lib.binding().rmsnorm_fwd(x, weight, eps, residual, out_dtype, mx_bits, had_block, out, want_rstd)
    if done is not None:
        return _result(done)
    name = "quest_rmsnorm_fwd"
    out = dict(out or {})
    _beside(name, x, weight=weight, residual=residual, **{k: out.get(k) for k in ("h", "rstd", "y", "yq", "sy")})
    ldx, (rows, cols) = _rows_of(name, "x", x), x.shape
    if tuple(weight.shape) != (cols,) or not weight.is_contiguous():
        raise ValueError(f"{name}: weight must be a contiguous vector of {cols} elements")
    ldr = cols
    if residual is not None:
        ldr = _rows_of(name, "residual", residual, x.shape)
        if residual.dtype != x.dtype:
            raise TypeError(f"{name}: x and residual share one dtype")
    if mx_bits is not None:
        _mx_check(name, mx_bits)
    with torch.cuda.device(x.device):
        if residual is not None:
            _kept(name, out, "h", (rows, cols), x.dtype, x.device)
        else:
            out["h"] = None
        if want_rstd or out.get("rstd") is not None:
            _kept(name, out, "rstd", (rows,), torch.float32, x.device)
        else:
            out["rstd"] = None
        ydt = F32
        if mx_bits is not None:
            _kept(name, out, "yq", (rows, cols * mx_bits // 8), torch.uint8, x.device)
            _kept(name, out, "sy", (quest_mx_scales_bytes(rows, cols),), torch.uint8, x.device)
        else:
            dt = out["y"].dtype if out.get("y") is not None else out_dtype or x.dtype
            ydt = _dtype_code(_kept(name, out, "y", (rows, cols), dt, x.device))
        _lib.check(_lib.load().quest_rmsnorm_fwd(
            _p(x), _p(residual), _dtype_code(x), ldx, ldr, _p(weight), _dtype_code(weight), rows, cols, ctypes.c_float(eps),
            _p(out["h"]), _p(out["rstd"]), _p(out["y"]) if mx_bits is None else None, ydt, mx_bits or 0, had_block,
            _p(out["yq"]) if mx_bits else None, _p(out["sy"]) if mx_bits else None, _stream()))
    return out


def quest_rmsnorm_bwd_workspace_bytes(rows: int, cols: int) -> int:
    return int(_lib.load().quest_rmsnorm_bwd_workspace_bytes(rows, cols))


def quest_rmsnorm_bwd(dy: torch.Tensor, h: torch.Tensor, weight: torch.Tensor, rstd: torch.Tensor, dres: torch.Tensor = None,
                      out: dict = None, want_dx: bool = True, want_dw: bool = True, workspace: torch.Tensor = None) -> dict:
    """Gradient of ``quest_rmsnorm_fwd``: ``h`` is what was normalised (the forward call's "h", or x without a residual),
    ``dres`` the gradient that reaches h on the residual stream.  Returns {"dx": the gradient of x and of the residual, "dw":
    float32 [cols]}; ``out`` may hold preallocated tensors under those keys, "dx" may be ``dy``, ``h`` or ``dres`` itself."""
    done = _lib.binding().rmsnorm_bwd(dy, h, weight, rstd, dres, out, want_dx, want_dw, workspace)
    if done is not None:
        return _result(done)
    name = "quest_rmsnorm_bwd"
    out = dict(out or {})
    _beside(name, dy, h=h, weight=weight, rstd=rstd, dres=dres, workspace=workspace, **{k: out.get(k) for k in ("dx", "dw")})
    lddy, (rows, cols) = _rows_of(name, "dy", dy), dy.shape
    ldh, lddr = _rows_of(name, "h", h, dy.shape), cols
    if dres is not None:
        lddr = _rows_of(name, "dres", dres, dy.shape)
    if h.dtype != dy.dtype or (dres is not None and dres.dtype != dy.dtype):
        raise TypeError(f"{name}: dy, h and dres share one dtype")
    if tuple(weight.shape) != (cols,) or not weight.is_contiguous():
        raise ValueError(f"{name}: weight must be a contiguous vector of {cols} elements")
    if rstd.dtype != torch.float32 or not rstd.is_contiguous() or rstd.numel() < rows:
        raise ValueError(f"{name}: rstd must be a contiguous float32 tensor of {rows} elements")
    want_dx, want_dw = want_dx or out.get("dx") is not None, want_dw or out.get("dw") is not None
    with torch.cuda.device(dy.device):
        for key, wanted, shape, dt in (("dx", want_dx, (rows, cols), dy.dtype), ("dw", want_dw, (cols,), torch.float32)):
            if wanted:
                _kept(name, out, key, shape, dt, dy.device)
            else:
                out[key] = None
        if workspace is None and want_dw:
            workspace = torch.empty(quest_rmsnorm_bwd_workspace_bytes(rows, cols), dtype=torch.uint8, device=dy.device)
        _lib.check(_lib.load().quest_rmsnorm_bwd(
            _p(dy), _p(h), _p(dres), _dtype_code(dy), lddy, ldh, lddr, _p(weight), _dtype_code(weight), _p(rstd), rows, cols,
            _p(out["dx"]), _p(out["dw"]), _p(workspace), _workspace_bytes_of(name, workspace), _stream()))
    return out
