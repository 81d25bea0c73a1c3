"""Timing cases of the microscaled (MX) layer and of the normalisation in front of it.

An MX tensor holds rows of 4-bit (E2M1) or 8-bit (E4M3) elements with one power-of-two scale, a UE8M0 byte, for every 32
consecutive elements of a row.  ``listed()`` names the standing cases, ``draw(rng)`` makes one more of the same ranges,
``prepare`` builds what a program holds before the call, ``run`` makes one pass (through the package's entry points where
``own`` is true, in elementary torch operations otherwise), ``work`` counts what the pass cannot do without, ``exact``
gives the same outputs in binary64.

Kinds of work:

  quantize   a bfloat16 or binary32 tensor to MX and back: weights when a model is loaded, activations kept in 8 bits.
  linear     an inference layer: weights in 4-bit MX from a checkpoint, laid out when the model was loaded; activations
             are quantized in the call.
  train      a layer's training step: x and w quantized, product, both gradients (straight through the rounding).
  norm       RMS norm of x + residual: the new residual stream and the normalised rows, as they are or in 8-bit MX.
  norm_bwd   its gradient with respect to the stream and to the weight.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f32": 4}
_BLOCK = 32                     # elements under one scale
_EPS = 1e-5


def _case(name, kind, M, K, N=0, bits=8, g=1, dtype="bf16", out="bf16", residual=False):
    return {"name": name, "kind": kind, "M": M, "N": N, "K": K, "bits": bits, "g": g, "dtype": dtype, "out": out,
            "residual": residual}


def listed():
    return [
        # model load: the gate or up weights of the 1.6B-scale MLP to 4 bits, blocks of 32 rotated
        _case("quantize_weights", "quantize", 5504, 2048, bits=4, g=32),
        # a large batch of activations kept in 8 bits
        _case("quantize_activations", "quantize", 16384, 4096, bits=8),
        # one token of one sequence through an attention projection: the smallest call, made for every layer and token
        _case("decode_one_token", "linear", 1, 2048, 2048, bits=8, g=32),
        # one step of 24 sequences through the gate or up projection
        _case("decode_batch", "linear", 24, 2048, 5504, bits=8, g=32),
        # a prompt of odd length through the down projection
        _case("prefill_ragged", "linear", 777, 5504, 2048, bits=8),
        # a large prefill with 4-bit activations
        _case("prefill_w4a4", "linear", 16384, 4096, 4096, bits=4, g=32),
        # a training step of the headline layer, both operands in 4 bits
        _case("train_w4a4", "train", 4096, 2048, 2048, bits=4, g=32),
        # a short batch through the MLP width with 8-bit activations, gradients in binary32 for an optimizer
        _case("train_w4a8_f32", "train", 512, 2048, 5504, bits=8, out="f32"),
        # one token before a projection: the stream's addition, the norm and the 8-bit activations
        _case("norm_one_token", "norm", 1, 2048, out="mx8", residual=True),
        # a training batch: bfloat16 rows out
        _case("norm_batch", "norm", 8192, 2048, residual=True),
        # the gradient for that batch, with the gradient that arrives on the residual stream
        _case("norm_bwd_batch", "norm_bwd", 8192, 2048, residual=True),
        # a binary32 model at the MLP width, odd number of rows, first norm of a stack (no stream gradient)
        _case("norm_bwd_f32_ragged", "norm_bwd", 777, 5504, dtype="f32"),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _multiple(rng, lo, hi, step):
    return max(lo, min(hi, int(round(_log_uniform(rng, lo, hi) / step)) * step))


def draw(rng):
    kind = rng.choice(["quantize", "linear", "linear", "linear", "train", "norm", "norm", "norm_bwd"])
    while True:
        # row lengths: hidden sizes and MLP widths, multiples of 128 as models have them, now and then of 32 only
        K = _multiple(rng, 256, 5504, 128 if rng.random() < 0.8 else 32)
        N = _multiple(rng, 256, 5504, 128 if rng.random() < 0.7 else 8)
        M = int(_log_uniform(rng, 1, 16384))
        bits, g = rng.choice([4, 8, 8]), rng.choice([1, 32])
        dtype, out, residual = "bf16", "bf16", False
        if kind == "quantize":
            M, N = int(_log_uniform(rng, 64, 16384)), 0
            dtype = rng.choice(["bf16", "bf16", "f32"])
        elif kind == "linear":
            if rng.random() < 0.4:
                M = int(_log_uniform(rng, 1, 33))
            dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
            # rotated rows are rounded after binary32 sums: there the type of y is the wider of the two errors
            out = rng.choice(["bf16", "bf16", "f32"]) if g == 1 else "bf16"
        elif kind == "train":
            M, N = _multiple(rng, 64, 8192, 8), N // 8 * 8
            out = rng.choice(["bf16", "f32"]) if g == 1 else "bf16"
        else:
            N, bits, g = 0, 8, 1
            if rng.random() < 0.3:
                K = int(_log_uniform(rng, 64, 8192))          # rows that no vector access divides
            dtype, residual = rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.7
            out = dtype
            if kind == "norm" and K % _BLOCK == 0 and rng.random() < 0.5:
                out = "mx8"
        if kind in ("linear", "train") and bits == 8:
            K = max(256, K // 128 * 128)                      # 8-bit rows meet 4-bit rows in whole groups of 128
        case = {"kind": kind, "M": M, "N": N, "K": K, "bits": bits, "g": g, "dtype": dtype, "out": out, "residual": residual}
        w = work(case)
        if w["flops"] <= (110e9 if kind == "train" else 550e9) and w["bytes"] <= 260e6:
            return case


# ---- inputs ------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) & 0x7FFFFFFFFFFFFFFF)
    return g


def _randn(shape, gen):
    return torch.randn(shape, generator=gen, device="cuda")


def _activations(rows, cols, gen, dtype):
    """Student-t with four degrees of freedom, as hidden activations of a trained transformer are heavy-tailed."""
    chi = torch.zeros((rows, cols), device="cuda")
    for _ in range(4):
        chi += _randn((rows, cols), gen).square_()
    return _randn((rows, cols), gen).mul_(2.0).div_(chi.sqrt_()).to(dtype)


def _weights(rows, cols, gen, dtype):
    return _randn((rows, cols), gen).mul_(0.02).to(dtype)


def _scale_bytes(rows, cols):
    return -(-rows // 128) * -(-cols // 128) * 512


def prepare(case, seed):
    gen = _gen(seed)
    kind, M, N, K, bits, g = (case[k] for k in ("kind", "M", "N", "K", "bits", "g"))
    dt = _DTYPES[case["dtype"]]
    s = {"case": case, "x": _activations(M, K, gen, dt)}
    if kind == "linear":
        # the checkpoint's tensors, two E2M1 codes to a byte and one scale byte per 32 elements, and the scales in the
        # order in which the layer reads them: tiles of 128 rows x 4 scales, row r of a tile at 16 (r % 32) + 4 (r / 32)
        level, e = _mx_codes(_weights(N, K, gen, dt), 4, g)
        s["wq"] = level[:, 0::2] | level[:, 1::2] << 4
        s["w_scales"] = (e + 127).to(torch.uint8)
        room = torch.zeros((-(-N // 128) * 128, -(-K // 128) * 4), dtype=torch.uint8, device="cuda")
        room[:N, : K // _BLOCK] = s["w_scales"]
        s["sw"] = room.reshape(room.shape[0] // 128, 4, 32, -1, 4).permute(0, 3, 2, 1, 4).reshape(-1).contiguous()
        s["w_cached"] = {"wq": s["wq"], "sw": s["sw"]}
        s["y"] = torch.empty((M, N), dtype=_DTYPES[case["out"]], device="cuda")
        s["saved"] = {"xq": torch.empty((M, K * bits // 8), dtype=torch.uint8, device="cuda"),
                      "sx": torch.empty(_scale_bytes(M, K), dtype=torch.uint8, device="cuda")}
    elif kind == "train":
        s["w"] = _weights(N, K, gen, dt)
        s["dy"] = _randn((M, N), gen).mul_(1e-3).to(torch.bfloat16)
    elif kind in ("norm", "norm_bwd"):
        s["weight"] = (1.0 + 0.1 * _randn((K,), gen)).to(dt)
        if kind == "norm" and case["residual"]:
            s["residual"] = _activations(M, K, gen, dt)
        if kind == "norm_bwd":
            # what the forward pass left: x is the stream that was normalised, rstd its rows' factors
            s["rstd"] = (s["x"].double().square().mean(1) + _EPS).rsqrt().float()
            s["dy"] = _randn((M, K), gen).mul_(1e-3).to(dt)
            if case["residual"]:
                s["dres"] = _randn((M, K), gen).mul_(1e-3).to(dt)
    return s


# ---- the operators in elementary operations, 32 bits ---------------------------------------------------

def _rotate32(v, g):
    """Orthonormal Walsh-Hadamard transform of blocks of g elements, strides from g/2 down to 1, every sum rounded."""
    if g == 1:
        return v
    shape, h = v.shape, g // 2
    while h:
        v = v.reshape(-1, g // (2 * h), 2, h)
        v = torch.stack((v[..., 0, :] + v[..., 1, :], v[..., 0, :] - v[..., 1, :]), dim=-2)
        h //= 2
    return v.reshape(shape) * (1.0 / math.sqrt(g))


_TOP = {4: 2, 8: 8}             # exponent of the largest element: E2M1 6 = 1.5 * 2^2, E4M3 448 = 1.75 * 2^8


def _power(e):
    """2^e in binary32, e in -127 .. 127: the exponent's bits, and the subnormal 2^-127."""
    return ((e.int() + 127) << 23).clamp_min(1 << 22).view(torch.float32)


def _mx_scaled(v, bits):
    """(v over its block's scale, scale exponents [rows, cols / 32])."""
    b = v.reshape(v.shape[0], -1, _BLOCK)
    amax = b.abs().amax(-1)
    e = (torch.frexp(amax).exponent - 1 - _TOP[bits]).clamp(-127, 127)
    e = torch.where(amax == 0, -127, e)
    return (b * _power(-e)[..., None]).reshape(v.shape), e


def _mx_codes(x, bits, g):
    """E2M1 codes (one to a byte) or E4M3 values, and scale exponents, of the rows of x."""
    t, e = _mx_scaled(_rotate32(x.float(), g), bits)
    if bits == 8:
        return t.clamp(-448.0, 448.0).to(torch.float8_e4m3fn), e
    # E2M1 magnitudes 0 .5 1 1.5 2 3 4 6; a magnitude halfway between two goes to the even code
    a = t.abs()
    level = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)).to(torch.uint8)
    return level | torch.signbit(t).to(torch.uint8) << 3, e


def _mx_values(level, e, bits):
    """binary32 values of codes and scale exponents."""
    if bits == 8:
        v = level.float()
    else:
        grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=level.device)
        v = grid[(level & 7).long()] * (1.0 - 2.0 * (level >> 3).float())
    return (v.reshape(v.shape[0], -1, _BLOCK) * _power(e)[..., None]).reshape(v.shape)


def _mx(x, bits, g):
    return _mx_values(*_mx_codes(x, bits, g), bits)


def _plain(s):
    case = s["case"]
    kind, bits, g = case["kind"], case["bits"], case["g"]
    if kind == "quantize":
        return _mx(s["x"], bits, g).to(torch.bfloat16)
    if kind == "linear":
        level = torch.stack((s["wq"] & 15, s["wq"] >> 4), dim=-1).reshape(s["wq"].shape[0], -1)
        w = _mx_values(level, s["w_scales"].int() - 127, 4)
        return (_mx(s["x"], bits, g) @ w.T).to(_DTYPES[case["out"]])
    if kind == "train":
        x, w, dy, out = _mx(s["x"], bits, g), _mx(s["w"], 4, g), s["dy"].float(), _DTYPES[case["out"]]
        return {"y": (x @ w.T).to(s["x"].dtype), "dx": _rotate32(dy @ w, g).to(out), "dw": _rotate32(dy.T @ x, g).to(out)}
    if kind == "norm":
        h = s["x"].float()
        if case["residual"]:
            h = (h + s["residual"].float()).to(s["x"].dtype).float()      # the stream is stored in its own type
        rstd = (h.square().mean(1) + _EPS).rsqrt()
        y = h * rstd[:, None] * s["weight"].float()
        y = _mx(y, 8, 1).to(torch.bfloat16) if case["out"] == "mx8" else y.to(_DTYPES[case["out"]])
        return {"h": h.to(s["x"].dtype) if case["residual"] else None, "rstd": rstd, "y": y}
    xhat, dy = s["x"].float() * s["rstd"][:, None], s["dy"].float()
    wdy = dy * s["weight"].float()
    dx = (wdy - xhat * (wdy * xhat).mean(1, keepdim=True)) * s["rstd"][:, None]
    if case["residual"]:
        dx = dx + s["dres"].float()
    return {"dx": dx.to(s["x"].dtype), "dw": (dy * xhat).sum(0)}


def run(state):
    if not own:
        return _plain(state)
    import paper_2502_05003_b200 as quest
    s, case = state, state["case"]
    kind, bits, g, K = case["kind"], case["bits"], case["g"], case["K"]
    if kind == "quantize":
        codes, scales = quest.quest_quantize_mx(s["x"], bits, g)
        return quest.quest_dequantize_mx(codes, scales, bits)
    if kind == "linear":
        return quest.quest_linear_fwd_mx(s["x"], None, bits, g, y=s["y"], saved=s["saved"], w_cached=s["w_cached"],
                                         want_codes=False)["y"]
    if kind == "train":
        r = quest.quest_linear_fwd_mx(s["x"], s["w"], bits, g)
        d = quest.quest_linear_bwd_mx(s["dy"], r, bits, g, K, out_dtype=_DTYPES[case["out"]])
        return {"y": r["y"], "dx": d["dx"], "dw": d["dw"]}
    if kind == "norm":
        if case["out"] == "mx8":
            r = quest.quest_rmsnorm_fwd(s["x"], s["weight"], _EPS, residual=s.get("residual"), mx_bits=8)
            y = quest.quest_dequantize_mx(r["yq"], r["sy"], 8)
        else:
            r = quest.quest_rmsnorm_fwd(s["x"], s["weight"], _EPS, residual=s.get("residual"))
            y = r["y"]
        return {"h": r["h"], "rstd": r["rstd"], "y": y}
    return quest.quest_rmsnorm_bwd(s["dy"], s["x"], s["weight"], s["rstd"], dres=s.get("dres"))


# ---- what a pass cannot do without ---------------------------------------------------------------------

def _mx_bytes(rows, cols, bits):
    return rows * cols * bits / 8 + rows * cols / _BLOCK


def work(case):
    kind, M, N, K, bits = (case[k] for k in ("kind", "M", "N", "K", "bits"))
    e = _SIZE[case["dtype"]]
    if kind == "quantize":
        # the tensor in, codes and scales out, and the bfloat16 values that are read back from them
        return {"bytes": M * K * (e + 2.0) + 2 * _mx_bytes(M, K, bits), "flops": M * K * (4.0 + math.log2(case["g"]))}
    if kind == "linear":
        return {"bytes": M * K * e + _mx_bytes(N, K, 4) + float(M * N * _SIZE[case["out"]]), "flops": 2.0 * M * N * K}
    if kind == "train":
        o = _SIZE[case["out"]]
        return {"bytes": (M + N) * K * (e + o) + M * N * (e + 2.0), "flops": 6.0 * M * N * K}
    if kind == "norm":
        y = _mx_bytes(M, K, 8) * 2 + 2 * M * K if case["out"] == "mx8" else M * K * e
        return {"bytes": M * K * e * (3 if case["residual"] else 1) + y + K * e + 4.0 * M, "flops": 5.0 * M * K}
    return {"bytes": M * K * e * (4 if case["residual"] else 3) + K * (e + 4.0) + 4.0 * M, "flops": 10.0 * M * K}


# ---- the same outputs in binary64 ----------------------------------------------------------------------

def _hadamard64(g):
    i = torch.arange(g, device="cuda")
    both = i[:, None] & i[None, :]
    odd = sum((both >> b) & 1 for b in range(6)) % 2
    return (1.0 - 2.0 * odd.double()) / math.sqrt(g)


def _turned64(v, g):
    return v if g == 1 else (v.reshape(-1, g) @ _hadamard64(g)).reshape(v.shape)


def _two64(e):
    """2^e in binary64 from the bits of its exponent: many values lie halfway between two elements."""
    return (e.long() + 1023 << 52).view(torch.float64)


def _micro64(v, bits):
    """Every block of 32 over 2^(floor(log2 max) - emax), rounded to the element type's nearest number, and back."""
    b = v.double().reshape(v.shape[0], -1, _BLOCK)
    most = b.abs().amax(-1, keepdim=True)
    scale = _two64((torch.frexp(most).exponent - 1 - _TOP[bits]).clamp(-127, 127))
    q = b / scale
    low, digits, most_q = (0, 1, 6.0) if bits == 4 else (-6, 3, 448.0)
    step = _two64((torch.frexp(q).exponent - 1).clamp(low, 16) - digits)
    return ((q / step).round() * step).clamp(-most_q, most_q).mul(scale).reshape(v.shape)


def exact(case, seed):
    gen = _gen(seed)
    kind, M, N, K, bits, g = (case[k] for k in ("kind", "M", "N", "K", "bits", "g"))
    dt = _DTYPES[case["dtype"]]
    x = _activations(M, K, gen, dt)
    if kind == "quantize":
        return _micro64(_turned64(x.double(), g), bits)
    if kind in ("linear", "train"):
        # the weights' codes are inputs of an inference layer: they are rounded from binary32 sums as the checkpoint's were
        w = _weights(N, K, gen, dt)
        if kind == "linear":
            wq = _mx_values(*_mx_codes(w, 4, g), 4).double()
        else:
            wq = _micro64(_turned64(w.double(), g), 4)
        xq = _micro64(_turned64(x.double(), g), bits)
        if kind == "linear":
            return xq @ wq.T
        dy = _randn((M, N), gen).mul_(1e-3).to(torch.bfloat16).double()
        return {"y": xq @ wq.T, "dx": _turned64(dy @ wq, g), "dw": _turned64(dy.T @ xq, g)}
    weight = (1.0 + 0.1 * _randn((K,), gen)).to(dt).double()
    if kind == "norm":
        h = x.double()
        if case["residual"]:
            h = (h + _activations(M, K, gen, dt).double()).to(dt).double()
        rstd = 1.0 / torch.sqrt((h * h).sum(1) / K + _EPS)
        y = h * weight * rstd[:, None]
        return {"h": h if case["residual"] else None, "rstd": rstd, "y": _micro64(y, 8) if case["out"] == "mx8" else y}
    rstd = (x.double().square().mean(1) + _EPS).rsqrt().float().double()
    dy = _randn((M, K), gen).mul_(1e-3).to(dt).double()
    dres = _randn((M, K), gen).mul_(1e-3).to(dt).double() if case["residual"] else 0.0
    n = x.double() * rstd[:, None]
    inner = torch.einsum("ij,ij,j->i", dy, n, weight) / K
    return {"dx": dres + rstd[:, None] * (dy * weight - n * inner[:, None]), "dw": torch.einsum("ij,ij->j", dy, n)}
