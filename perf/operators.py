"""The microscaled operators whose speed is measured, and their plain forms.

MX numbers: 32 consecutive elements of a row share a scale 2^e (E8M0); an element
is a 4-bit float (E2M1, "fp4") or an 8-bit one (E4M3, "fp8"). Sizes are those of
the repository's workloads (the Llama-70B MLP, 8192 x 28672 x 8192, and the
Granite-20B MLP, 6144 x 24576 x 6144, at their tensor-parallel degrees) or generic.

A case holds
  op      "quantize" (mx_quantize; fp4 codes come back through mx_dequantize),
          "norm" (rmsnorm), "gemm" (mx_gemm) or "mlp" (mx_mlp_shard)
  M, K    rows and columns of X (for a weight being quantized: its outputs and inputs)
  N, N2   gemm, mlp: outputs of the first weight and of the second one
  fmt     "fp8" or "fp4" codes of X or of what is quantized; norm also "none", 16 bits
  dtype   "bf16" or "fp16" of the tensors in 16 bits
  residual  norm: X is added to a residual first
  gated   mlp: silu(gate) * up, else the up projection alone
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5


def _case(name, op, M, K, N=0, N2=0, fmt="fp8", dtype="bf16", residual=False, gated=False):
    c = dict(op=op, M=M, K=K, N=N, N2=N2, fmt=fmt, dtype=dtype, residual=residual, gated=gated)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest call: one token's activations before a product
        _case("quantize_m1", "quantize", 1, 8192),
        # a short ragged prompt's activations
        _case("quantize_ragged_m777", "quantize", 777, 5000, dtype="fp16"),
        # a model being converted: a whole Llama-70B layer to 4 bits and back, to see what it loses
        _case("quantize_weight", "quantize", 28672, 8192, fmt="fp4"),
        # token generation: residual, norm and 8-bit activations of one token
        _case("norm_m1", "norm", 1, 8192, residual=True),
        # a prompt of 1000 tokens before a W4A16 layer, 16 bits in and out
        _case("norm_m1000", "norm", 1000, 6144, fmt="none", dtype="fp16", residual=True),
        # prefill of a long prompt
        _case("norm_m2048", "norm", 2048, 8192, residual=True),
        # token generation for one sequence: one projection of Llama-70B at TP = 8
        _case("gemm_m1", "gemm", 1, 8192, 3584),
        # a short ragged prompt; odd sizes
        _case("gemm_ragged_m77", "gemm", 77, 5000, 3464, dtype="fp16"),
        # a full serving batch on one GPU that holds the whole Llama-70B layer, 4-bit activations
        _case("gemm_unsharded_m64", "gemm", 64, 8192, 28672, fmt="fp4"),
        # prefill of a long prompt, Llama-70B at TP = 2
        _case("gemm_m2048", "gemm", 2048, 8192, 14336),
        # token generation for a batch of 16: the gated MLP of Llama-70B at TP = 8
        _case("mlp_m16", "mlp", 16, 8192, 3584, 8192, gated=True),
        # a prompt of 1000 tokens through the same MLP
        _case("mlp_m1000", "mlp", 1000, 8192, 3584, 8192, gated=True),
    ]


def _log_uniform(rng, lo, hi, step):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    """Another case of the ranges above: 1 to 2048 tokens, rows and columns from 512 to 16384 (most of them
    whole tiles, some ragged), all formats and types. Costs are bounded by the largest listed case."""
    op = rng.choice(["quantize", "norm", "gemm", "gemm", "mlp", "mlp"])
    dtype = rng.choice(["bf16", "fp16"])
    step = rng.choice([8, 128, 128, 128])  # one in four ragged
    K = _log_uniform(rng, 512, 16384, step)
    if op == "quantize":
        return _case(None, op, _log_uniform(rng, 1, 8192, 1), K, fmt=rng.choice(["fp8", "fp4"]), dtype=dtype)
    if op == "norm":
        return _case(None, op, _log_uniform(rng, 1, 4096, 1), K, fmt=rng.choice(["fp8", "fp8", "none"]), dtype=dtype,
                     residual=rng.random() < 0.75)
    N = _log_uniform(rng, 512, 16384, step)
    N2 = _log_uniform(rng, 512, 8192, 128) if op == "mlp" else 0
    gated = op == "mlp" and rng.random() < 0.7
    M = _log_uniform(rng, 1, 2048, 1)
    flops = 2 * M * (K * N * (1 + gated) + N * N2)
    if flops > 450e9:
        M = max(1, int(M * 450e9 / flops))
    return _case(None, op, M, K, N, N2, fmt=rng.choice(["fp8", "fp8", "fp4"]), dtype=dtype, gated=gated)


def _packed(K, fmt):
    """Bytes of a row of K codes."""
    return -(-K // 32) * (16 if fmt == "fp4" else 32)


def work(case):
    c = case
    M, K, N = c["M"], c["K"], c["N"]
    x = M * (_packed(K, c["fmt"]) + -(-K // 32))
    w = N * (_packed(K, "fp4") + -(-K // 32))
    if c["op"] == "quantize":  # fp4: the values come back in 16 bits
        return {"bytes": 2 * M * K + (2 * M * K if c["fmt"] == "fp4" else x), "flops": 2 * M * K}
    if c["op"] == "norm":
        return {"bytes": 2 * M * K * (3 if c["residual"] else 1) + 2 * K + (2 * M * K if c["fmt"] == "none" else x),
                "flops": 6 * M * K}
    if c["op"] == "gemm":
        return {"bytes": x + w + 2 * M * N, "flops": 2 * M * N * K}
    down = c["N2"] * (_packed(N, "fp4") + -(-N // 32))
    firsts = 2 if c["gated"] else 1
    return {"bytes": x + firsts * w + down + 2 * M * c["N2"], "flops": 2 * M * N * (firsts * K + c["N2"])}


# ---- inputs --------------------------------------------------------------

def _activations(g, M, K, dtype):
    """Normal values times a factor for each channel, a few channels far above the rest, as a transformer's
    residual stream has them."""
    channel = torch.exp(0.5 * torch.randn(K, generator=g, device="cuda"))
    channel = torch.where(torch.rand(K, generator=g, device="cuda") < 0.002, 20 * channel, channel)
    return (torch.randn(M, K, generator=g, device="cuda") * channel).to(dtype)


def _mx_weight(g, N, K):
    """Codes [N][ceil(K/32) * 16], two to a byte (the even column in the low half), and scales 2^(s - 127)
    [N][ceil(K/32)]; uniform codes, zero past K."""
    blocks = -(-K // 32)
    codes = torch.randint(0, 256, (N, blocks * 16), generator=g, device="cuda", dtype=torch.uint8)
    codes[:, K // 2:] = 0
    return codes, torch.randint(116, 120, (N, blocks), generator=g, device="cuda", dtype=torch.uint8)


def prepare(case, seed):
    c, dt = case, DTYPES[case["dtype"]]
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    M, K = c["M"], c["K"]
    state = {"case": c, "x": _activations(g, M, K, dt)}
    if c["op"] == "norm":
        state["weight"] = (1 + 0.2 * torch.randn(K, generator=g, device="cuda")).to(dt)
        state["residual"] = _activations(g, M, K, dt) if c["residual"] else None
    if c["op"] in ("gemm", "mlp"):  # X as the layer before leaves it, weights as a checkpoint holds them
        state["x"] = _quantize(state["x"].float(), c["fmt"])
        shapes = [(c["N"], K)] * (2 if c["gated"] else 1) + ([(c["N2"], c["N"])] if c["op"] == "mlp" else [])
        state["w"] = [_mx_weight(g, *s) for s in shapes]
    if own:  # what a program keeps: the activations' handle, and the weights in the order the product reads
        import paper_2402_04925_amd as tpdq
        state["tpdq"], state["fmt"] = tpdq, {"fp4": tpdq.MX_FP4, "fp8": tpdq.MX_FP8, "none": None}[c["fmt"]]
        if c["op"] in ("gemm", "mlp"):
            state["x"] = tpdq.MxTensor.from_tensors(*state["x"], K, state["fmt"])
            inner = [K] * (2 if c["gated"] else 1) + [c["N"]]
            state["w"] = [tpdq.mx_pack(tpdq.MxTensor.from_tensors(*w, k, tpdq.MX_FP4))
                          for w, k in zip(state["w"], inner)]
    return state


# ---- plain forms ---------------------------------------------------------

def _quantize(x, fmt):
    """x fp32 [M][K] -> (codes, scales): fp8 codes float8_e4m3fn [M][ceil(K/32) * 32], fp4 codes packed two to
    a byte; scales uint8, 2^(s - 127)."""
    M, K = x.shape
    x = torch.nn.functional.pad(x, (0, -K % 32)).view(M, -1, 32)
    top = x.abs().amax(-1)
    e = torch.frexp(top).exponent - 1 - (2 if fmt == "fp4" else 8)
    e = torch.where(top == 0, -127, e).clamp(-127, 127)
    v = torch.ldexp(x, -e.unsqueeze(-1)).view(M, -1)
    scales = (e + 127).to(torch.uint8)
    if fmt == "fp8":
        return v.clamp(-448, 448).to(torch.float8_e4m3fn), scales
    a = v.abs()
    code = ((a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte()
            + (a >= 3.5).byte() + (a > 5).byte() + 8 * (v < 0).byte())
    return code[:, 0::2] + 16 * code[:, 1::2], scales


def _values(codes, scales, K):
    """The numbers that codes and scales stand for, fp32 [M][K]."""
    if codes.dtype == torch.float8_e4m3fn:
        v = codes.float()
    else:
        one = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
        pairs = torch.stack([one.repeat(16), one.repeat_interleave(16)], dim=1)
        v = pairs[codes.int()].view(codes.shape[0], -1)
    v = torch.ldexp(v.view(codes.shape[0], -1, 32), (scales.int() - 127).unsqueeze(-1))
    return v.view(codes.shape[0], -1)[:, :K]


def _shown(codes, scales, K, dtype):
    """What a quantized result is returned as: fp8 elements and their scales; the values of fp4."""
    if codes.dtype == torch.float8_e4m3fn:
        return {"elements": codes[:, :K], "scales": scales.view(torch.float8_e8m0fnu)}
    return {"values": _values(codes, scales, K).to(dtype)}


def _product(x, w, K):
    return _values(*x, K) @ _values(*w, K).t()


def _plain(s):
    c, dt = s["case"], DTYPES[s["case"]["dtype"]]
    K, fmt = c["K"], c["fmt"]
    if c["op"] == "quantize":
        return _shown(*_quantize(s["x"].float(), fmt), K, dt)
    if c["op"] == "norm":
        h = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(dt)
        f = h.float()
        y = f * torch.rsqrt(f.square().mean(-1, keepdim=True) + EPS) * s["weight"].float()
        out = {"y": y.to(dt)} if fmt == "none" else _shown(*_quantize(y, fmt), K, dt)
        return out if s["residual"] is None else dict(out, residual=h)
    if c["op"] == "gemm":
        return _product(s["x"], s["w"][0], K).to(dt)
    y1 = _product(s["x"], s["w"][0], K)
    if c["gated"]:
        y1 = y1 / (1 + torch.exp(-y1)) * _product(s["x"], s["w"][1], K)
    return _product(_quantize(y1, fmt), s["w"][-1], c["N"]).to(dt)


def _shown_own(q, s):
    K = s["case"]["K"]
    if s["fmt"] == s["tpdq"].MX_FP8:
        return {"elements": q.codes[:, :K], "scales": q.scales}
    return {"values": s["tpdq"].mx_dequantize(q, s["x"].dtype)}


def _own(s):
    c, tpdq = s["case"], s["tpdq"]
    dt = DTYPES[c["dtype"]]
    if c["op"] == "quantize":
        return _shown_own(tpdq.mx_quantize(s["x"], s["fmt"]), s)
    if c["op"] == "norm":
        y, h = tpdq.rmsnorm(s["x"], s["weight"], EPS, residual=s["residual"], fmt=s["fmt"])
        out = {"y": y} if s["fmt"] is None else _shown_own(y, s)
        return out if s["residual"] is None else dict(out, residual=h)
    if c["op"] == "gemm":
        return tpdq.mx_gemm(s["x"], s["w"][0], dt)
    return tpdq.mx_mlp_shard(s["x"], s["w"][-2], s["w"][-1], dt, w_gate=s["w"][0] if c["gated"] else None)


def run(state):
    return _own(state) if own else _plain(state)


# ---- the definition in 64 bits -------------------------------------------

def _exact_quantize(x, fmt):
    """x float64 [M][K] -> (elements, scales), both float64: elements on the format's grid, steps of 2^-1 (fp4)
    or 2^-3 (fp8) of the element's own power of two, which is at least the smallest normal one."""
    low, top, most, places = (0, 2, 6.0, 1) if fmt == "fp4" else (-6, 8, 448.0, 3)
    M, K = x.shape
    full = torch.zeros(M, -(-K // 32) * 32, dtype=torch.float64, device=x.device)
    full[:, :K] = x
    full = full.reshape(M, -1, 32)
    biggest = full.abs().max(dim=-1, keepdim=True).values
    scale = torch.exp2((torch.floor(torch.log2(biggest.clamp(min=2.0 ** -140))) - top).clamp(-127, 127))
    v = full / scale
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** low))) - places)
    v = (torch.round(v / step) * step).clamp(-most, most)
    return v.reshape(M, -1)[:, :K], scale.reshape(M, -1)


def _exact_values(codes, scales, K):
    if codes.dtype == torch.float8_e4m3fn:
        v = codes.double()
    else:
        c = torch.stack([codes % 16, codes // 16], dim=-1).reshape(codes.shape[0], -1)
        m = (c % 8).double()
        e = torch.floor(m / 2)
        v = torch.where(e == 0, m / 2, (1 + (m % 2) / 2) * torch.exp2(e - 1)) * (1 - 2 * (c >= 8).double())
    return (v * torch.exp2(scales.double() - 127).repeat_interleave(32, dim=1))[:, :K]


def exact(case, seed):
    c, s = case, prepare(case, seed)
    K, fmt = c["K"], c["fmt"]
    if own:
        return None
    if c["op"] in ("quantize", "norm"):
        y, more = s["x"].double(), {}
        if c["op"] == "norm":
            if s["residual"] is not None:
                more["residual"] = y = (y + s["residual"].double()).to(s["x"].dtype).double()
            y = y / torch.sqrt((y * y).sum(dim=1, keepdim=True) / K + EPS) * s["weight"].double()
            if fmt == "none":
                return dict(more, y=y)
        v, scale = _exact_quantize(y, fmt)
        if fmt == "fp8":
            return dict(more, elements=v, scales=scale)
        return {"values": v * scale.repeat_interleave(32, dim=1)[:, :K]}
    x = _exact_values(*s["x"], K)
    first = [x.matmul(_exact_values(*w, K).T.contiguous()) for w in s["w"][:2 if c["gated"] else 1]]
    if c["op"] == "gemm":
        return first[0]
    y1 = first[0] * torch.sigmoid(first[0]) * first[1] if c["gated"] else first[0]
    v, scale = _exact_quantize(y1, fmt)
    y1 = v * scale.repeat_interleave(32, dim=1)[:, :c["N"]]
    return y1.matmul(_exact_values(*s["w"][-1], c["N"]).T.contiguous())
