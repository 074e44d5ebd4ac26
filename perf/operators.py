"""Layers whose activations have 8 or 16 bits, against the library's packed 4-bit weights, as cases that can be timed and checked.

* "quantize": activations -> MXFP8 (E4M3 elements, one power-of-two scale per 32 channels), reordered for the packed weights.
* "norm": the residual's addition and RMSNorm in front of it; the sum goes on as the new hidden state.
* "gemm": MXFP8 activations times packed MXFP4 weights.  Weights packed with S outlier copies for the 4-bit path serve it as they are.
* "gemv", "mx_gemv": a few fp16 rows, straight from the layer before, times packed NVFP4 / MXFP4 weights.

Where `own` is true `run` calls the library; otherwise it computes the same in elementary torch operations, in 32 bits, on the packed
operands.  `exact` goes by the definitions in 64 bits.
"""
import math

import torch

#: The library's calls, or the plain forms.
own = False

#: A drawn product has at most this many multiplications, the largest listed one's, and this many weights.
MOST = 8192 * 8192 * 28672
MOST_WEIGHTS = 8192 * 28672
#: Bytes of the scratch memory that a program keeps for the calls that take some.
SCRATCH = 64 << 20


def _case(name, op, M, K, N=0, S=0, perm=True, up=False, residual=False, pad=0, out="f16"):
    return {"name": name, "op": op, "M": M, "K": K, "N": N, "S": S, "perm": perm, "up": up, "residual": residual, "pad": pad, "out": out}


def listed():
    return [
        # one token into the down projection of an 8B model: latency
        _case("quantize_1x14336", "quantize", 1, 14336),
        # 8192 tokens into the down projection of a 70B model: the largest stream
        _case("quantize_8192x28672", "quantize", 8192, 28672, up=True),
        # one token behind the attention of an 8B model: latency
        _case("norm_1x4096", "norm", 1, 4096, residual=True),
        # a short prompt of a 32B model, rows as they come, hidden states inside a wider buffer, channels in their own order
        _case("norm_333x5120", "norm", 333, 5120, perm=False, residual=True, pad=64),
        # a prompt of 2048 tokens of a 70B model
        _case("norm_2048x8192", "norm", 2048, 8192, residual=True),
        # 16 users decoding, up projection of an 8B model
        _case("gemm_16x4096x14336", "gemm", 16, 4096, 14336),
        # a prompt with rows and features as they come, weights packed for the 4-bit path too, fp32 output
        _case("gemm_777x4352x6147_f32", "gemm", 777, 4352, 6147, S=224, out="f32"),
        # the largest: down projection of a 70B model over 8192 tokens
        _case("gemm_8192x28672x8192", "gemm", 8192, 28672, 8192),
        # one token of one user: query projection of an 8B model, the smallest product
        _case("gemv_1x4096x4096", "gemv", 1, 4096, 4096, S=256),
        # seven users, down projection of a 70B model
        _case("gemv_7x28672x8192", "gemv", 7, 28672, 8192, S=1024, out="f32"),
        # one user, gate projection of a 32B model, channels in their own order
        _case("mx_gemv_1x5120x27648", "mx_gemv", 1, 5120, 27648, perm=False),
        # sixteen users, down projection of an 8B model
        _case("mx_gemv_16x14336x4096", "mx_gemv", 16, 14336, 4096, S=256),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "norm", "gemm", "gemm", "gemv", "mx_gemv"])
    unit = 16 if op == "gemv" else 32
    K = max(unit, _log(rng, 256, 28672) // unit * unit)
    perm = rng.random() < 0.7
    if op in ("quantize", "norm"):
        M = min(_log(rng, 1, 16384), 8192 * 28672 // K)
        pad = rng.choice([0, 0, 8, 64])
        c = _case("", op, M, K, perm=perm, up=rng.random() < 0.3, residual=op == "norm" and rng.random() < 0.8, pad=pad)
    else:
        N = min(_log(rng, 64, 32768), MOST_WEIGHTS // K)
        if rng.random() < 0.6:
            N = max(16, N // 16 * 16)
        M = _log(rng, 1, 8192) if op == "gemm" else _log(rng, 1, 32)
        M = max(1, min(M, MOST // (K * N)))
        S = rng.choice([0, min(K, _log(rng, unit, 1024) // unit * unit)])
        c = _case("", op, M, K, N, S=S, perm=perm, out=rng.choice(["f16", "f32"]), pad=0 if op == "gemm" else rng.choice([0, 8]))
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------------------------- inputs

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _rows(M, K, pad, factors, gen):
    """fp16 [M, K] inside rows of K + pad: normal values times a factor per channel."""
    buf = torch.zeros((M, K + pad), dtype=torch.float16, device="cuda")
    x = buf[:, :K]
    step = max(1, (64 << 20) // K)
    for r in range(0, M, step):
        n = min(step, M - r)
        x[r:r + n] = (torch.randn((n, K), device="cuda", generator=gen) * factors).clamp_(-60000.0, 60000.0).half()
    return x


def _factors(K, gen):
    """One channel of a hundred is 20 to 100 times as large as the others."""
    f = torch.ones(K, device="cuda")
    n = max(1, K // 100)
    at = torch.randperm(K, device="cuda", generator=gen)[:n]
    f[at] = torch.exp(torch.rand(n, device="cuda", generator=gen) * math.log(5.0) + math.log(20.0))
    return f


def _nibbles(v):
    """Nearest E2M1 codes of fp32 values, two a byte, the first in the low half."""
    bounds = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device="cuda")
    code = torch.bucketize(v.abs(), bounds, out_int32=True).to(torch.uint8) | (v < 0).to(torch.uint8) << 3
    return code[..., 0::2] | code[..., 1::2] << 4


def _weights(fmt, N, K, S, gen):
    """Packed weights [N, K + S] with the last S channels' blocks twice, N(0, 0.02): codes, scale bytes, tensor scale."""
    block = 16 if fmt == "gemv" else 32
    codes = torch.empty((N, (K + S) // 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty((N, (K + S) // block), dtype=torch.uint8, device="cuda")
    ts = 0.1 / 2688.0
    step = max(1, (64 << 20) // K)
    for r in range(0, N, step):
        n = min(step, N - r)
        w = (torch.randn((n, K // block, block), device="cuda", generator=gen) * 0.02).half().float()
        amax = w.abs().amax(-1)
        if fmt == "gemv":
            s8 = (amax / (6.0 * ts)).clamp(max=448.0).to(torch.float8_e4m3fn)
            s, byte = s8.float() * ts, s8.view(torch.uint8)
        else:
            e = torch.frexp(amax)[1] - 3
            s, byte = torch.ldexp(torch.ones_like(amax), e), (e + 127).to(torch.uint8)
        q = _nibbles((w / s.clamp(min=1e-30)[..., None]).reshape(n, K))
        codes[r:r + n, :K // 2], scales[r:r + n, :K // block] = q, byte
        if S:
            codes[r:r + n, K // 2:], scales[r:r + n, K // block:] = q[:, (K - S) // 2:], byte[:, (K - S) // block:]
    return codes, scales, ts


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    M, K, N, S = case["M"], case["K"], case["N"], case["S"]
    s = {"op": case["op"], "flags": 2 if case["up"] else 0, "perm": None, "residual": None}
    factors = _factors(K, gen)
    if case["perm"]:
        s["perm"] = torch.randperm(K, device="cuda", generator=gen).int()
    x = _rows(M, K, case["pad"], factors, gen)
    if case["op"] in ("quantize", "norm"):
        s["x"] = x
        s["codes"] = torch.empty((M, K), dtype=torch.uint8, device="cuda")
        s["scales"] = torch.empty((M, K // 32), dtype=torch.uint8, device="cuda")
        if case["op"] == "norm":
            s["gamma"] = (1.0 + 0.1 * torch.randn(K, device="cuda", generator=gen)).half()
            s["eps"] = 1e-5
            if case["residual"]:
                s["residual"] = _rows(M, K, case["pad"], factors, gen)
                s["hidden"] = torch.empty((M, K), dtype=torch.float16, device="cuda")
        return s
    s["w_codes"], s["w_scales"], s["ts"] = _weights(case["op"], N, K, S, gen)
    s["y"] = torch.empty((M, N), dtype=torch.float32 if case["out"] == "f32" else torch.float16, device="cuda")
    s["scratch"] = torch.empty(SCRATCH, dtype=torch.uint8, device="cuda")
    if case["op"] == "gemm":
        step = max(1, (64 << 20) // K)
        parts = [_mx8(x[r:r + step].float(), False) for r in range(0, M, step)]
        s["a_codes"], s["a_scales"] = (torch.cat([p[i] for p in parts]).view(torch.uint8) for i in range(2))
        s["perm"] = None
    else:
        s["x"] = x
    return s


# ------------------------------------------------------------------------------------------------------------ plain forms

def _mx8(v, up):
    """fp32 [M, K] -> E4M3 codes [M, K] and E8M0 scales [M, K / 32]."""
    M, K = v.shape
    b = v.reshape(M, K // 32, 32)
    m, e = torch.frexp(b.abs().amax(-1))
    e = e - 9 + (m > 0.875).int() if up else e - 9
    e = torch.where(m > 0, e, 0)
    q = torch.ldexp(b, -e[..., None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    return q.reshape(M, K), (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _fp4(codes, scales, K, block):
    """The first K columns of packed weights, in fp32, without the tensor scale."""
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=codes.device)
    c = codes[:, :K // 2].int()
    w = table[torch.stack((c & 15, c >> 4), -1).reshape(codes.shape[0], K // block, block)]
    s = scales[:, :K // block]
    s = s.view(torch.float8_e4m3fn).float() if block == 16 else torch.ldexp(torch.ones((), device=s.device), s.int() - 127)
    return (w * s[..., None]).reshape(-1, K)


def _plain(s):
    x, perm = s.get("x"), s["perm"]
    if s["op"] == "gemm":
        a = s["a_codes"].view(torch.float8_e4m3fn).float()
        M, K = a.shape
        a = torch.ldexp(a.reshape(M, K // 32, 32), s["a_scales"].int()[..., None] - 127).reshape(M, K)
        return (a @ _fp4(s["w_codes"], s["w_scales"], K, 32).T).to(s["y"].dtype)
    if s["op"] in ("gemv", "mx_gemv"):
        K = x.shape[1]
        v = (x if perm is None else x[:, perm]).float()
        if s["op"] == "gemv":
            return (v @ _fp4(s["w_codes"], s["w_scales"], K, 16).T * s["ts"]).to(s["y"].dtype)
        return (v @ _fp4(s["w_codes"], s["w_scales"], K, 32).T).to(s["y"].dtype)
    out = []
    if s["op"] == "norm":
        if s["residual"] is not None:
            x = (x.float() + s["residual"].float()).half()
            out = [x]
        mean = x.double().square().mean(-1, keepdim=True).float()
        x = (x.float() * (1.0 / torch.sqrt(mean + s["eps"]))).half() * s["gamma"]
    if perm is not None:
        x = x[:, perm]
    return [*_mx8(x.float(), s["flags"] != 0), *out]


def _library(s):
    from paper_2601_07475_amd import binding as B
    op = s["op"]
    if op == "gemm":
        return B.arcq_mx8_gemm(s["a_codes"], s["a_scales"], s["w_codes"], s["w_scales"], y=s["y"], workspace=s["scratch"])
    if op == "gemv":
        return B.arcq_gemv(s["x"], s["perm"], s["w_codes"], s["w_scales"], s["ts"], y=s["y"], workspace=s["scratch"])
    if op == "mx_gemv":
        return B.arcq_mx_gemv(s["x"], s["perm"], s["w_codes"], s["w_scales"], y=s["y"], workspace=s["scratch"])
    if op == "quantize":
        B.arcq_mx8_quantize_act(s["x"], s["perm"], s["flags"], codes=s["codes"], scales=s["scales"])
        hidden = []
    elif s["residual"] is None:
        B.arcq_mx8_add_rmsnorm_quantize_act(s["x"], None, s["gamma"], s["eps"], s["perm"], s["flags"], codes=s["codes"], scales=s["scales"])
        hidden = []
    else:
        B.arcq_mx8_add_rmsnorm_quantize_act(s["x"], s["residual"], s["gamma"], s["eps"], s["perm"], s["flags"], hidden=s["hidden"],
                                            codes=s["codes"], scales=s["scales"])
        hidden = [s["hidden"]]
    return [s["codes"].view(torch.float8_e4m3fn), s["scales"].view(torch.float8_e8m0fnu), *hidden]


def run(state):
    return _library(state) if own else _plain(state)


def work(case):
    M, K, N = case["M"], case["K"], case["N"]
    if case["op"] in ("quantize", "norm"):
        read = 2 * M * K * (2 if case["residual"] else 1) + (4 * K if case["perm"] else 0) + (2 * K if case["op"] == "norm" else 0)
        return {"bytes": read + M * K + M * K // 32 + (2 * M * K if case["residual"] else 0), "flops": (8 if case["op"] == "norm" else 3) * M * K}
    w = N * K // 2 + N * K // (16 if case["op"] == "gemv" else 32)
    a = M * K + M * K // 32 if case["op"] == "gemm" else 2 * M * K + (4 * K if case["perm"] else 0)
    return {"bytes": w + a + M * N * (4 if case["out"] == "f32" else 2), "flops": 2 * M * N * K}


# ------------------------------------------------------------------------------------------------ definitions, in 64 bits

def _exact_weights(codes, scales, K, block):
    low = (codes[:, :K // 2] & 15).long()
    high = (codes[:, :K // 2] // 16).long()
    values = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12, 0, -1, -2, -3, -4, -6, -8, -12], dtype=torch.float64, device=codes.device) / 2
    w = torch.empty((codes.shape[0], K), dtype=torch.float64, device=codes.device)
    w[:, 0::2], w[:, 1::2] = values[low], values[high]
    b = scales[:, :K // block].double()
    if block == 16:
        e, f = torch.floor(b / 8), b % 8
        scale = torch.where(e > 0, (1 + f / 8) * torch.exp2(e - 7), f * 2.0 ** -9)
    else:
        scale = torch.exp2(b - 127)
    w.reshape(-1, K // block, block).mul_(scale[..., None])
    return w


def _exact_mx8(v, up):
    """v fp64 [M, K] -> values of the codes and of the scales, fp64."""
    M, K = v.shape
    powers = torch.exp2(torch.arange(-160, 160, dtype=torch.float64, device=v.device))
    floor2 = lambda t: powers[(torch.searchsorted(powers, t.contiguous(), right=True) - 1).clamp(min=0)]  # noqa: E731
    b = v.reshape(M, K // 32, 32)
    amax = b.abs().amax(-1)
    scale = floor2(amax) / 256
    if up:
        scale = torch.where(amax > 448 * scale, 2 * scale, scale)
    scale = torch.where(amax > 0, scale, 1.0)
    q = (b / scale[..., None]).clamp(-448.0, 448.0)
    grid = floor2(q.abs()).clamp(min=2.0 ** -6) / 8
    return (torch.round(q / grid) * grid).reshape(M, K), scale


def exact(case, seed):
    s = prepare(case, seed)
    K, perm = case["K"], s["perm"]
    if case["op"] in ("gemm", "gemv", "mx_gemv"):
        if case["op"] == "gemm":
            a = s["a_codes"].view(torch.float8_e4m3fn).double().reshape(-1, K // 32, 32)
            a = (a * torch.exp2(s["a_scales"].double() - 127)[..., None]).reshape(-1, K)
        else:
            a = s["x"].double() if perm is None else s["x"].double()[:, perm.long()]
        w = _exact_weights(s["w_codes"], s["w_scales"], K, 16 if case["op"] == "gemv" else 32)
        return (a @ w.T) * (s["ts"] if case["op"] == "gemv" else 1.0)
    parts = []
    step = max(1, (16 << 20) // K)
    for r in range(0, case["M"], step):
        x, out = s["x"][r:r + step].double(), []
        if case["op"] == "norm":
            if case["residual"]:
                x = (x + s["residual"][r:r + step].double()).float().half().double()    # the sum of two fp16 values, rounded once
                out = [x]
            mean = x.square().mean(-1, keepdim=True).float()
            root = (mean.double() + float(torch.tensor(s["eps"]))).float().double().sqrt().float()
            rstd = (1.0 / root.double()).float()
            x = (x * rstd.double()).float().half().double() * s["gamma"].double()
            x = x.float().half().double()
        if perm is not None:
            x = x[:, perm.long()]
        parts.append([*_exact_mx8(x, case["up"]), *out])
    return [torch.cat(p) for p in zip(*parts)]
