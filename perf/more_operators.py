"""Whole layers on the library's packed 4-bit weights, as cases that can be timed and checked.

* "gemv", "mx_gemv": a few fp16 rows times packed NVFP4 / MXFP4 weights with bias, activation and residual: y = act(x W^T + bias) + residual.
* "mx8": the same behind MXFP8 activations times packed MXFP4 weights.
* "route": the router of a mixture of experts: fp16 rows times fp16 router weights, scores, the best experts of each token and their weights.
* "moe", "mx_moe": the experts for a few tokens: y[m] = sum of weight[m, j] (act(x G^T) * (x U^T)) D^T over the token's experts, + residual,
  on packed NVFP4 / MXFP4 weights: G over U in the rows of one operand, D in the other.

Where `own` is true `run` calls the library; otherwise it computes the same in elementary torch operations, in 32 bits (scores that experts are
chosen by in 64), on the packed operands.  `exact` goes by the definitions in 64 bits.
"""
import math

import torch

#: The library's calls, or the plain forms.
own = False

#: A drawn product has at most this many multiplications, the largest listed one's, and this many weights.
MOST = 4096 * 28672 * 8192
MOST_WEIGHTS = 8192 * 28672
#: Weights of all experts of a drawn layer, and weights times tokens that use them.
MOST_EXPERTS = 8 * 3 * 4096 * 14336
#: Bytes of the scratch memory that a program keeps for the calls.
SCRATCH = 64 << 20
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def _linear(name, op, M, K, N, S=0, bias=False, act="none", residual=False, perm=False, pad=0, out="f16"):
    return {"name": name, "op": op, "M": M, "K": K, "N": N, "S": S, "bias": bias, "act": act, "residual": residual, "perm": perm, "pad": pad, "out": out}


def _route(name, M, K, E, top, sigmoid=False, renorm=False, bias=False, pad=0):
    return {"name": name, "op": "route", "M": M, "K": K, "E": E, "top": top, "sigmoid": sigmoid, "renorm": renorm, "bias": bias, "pad": pad}


def _moe(name, op, M, K, I, E, top, S=0, S2=0, act="silu", residual=False, perm=False, drop=False, pad=0, out="f16"):
    return {"name": name, "op": op, "M": M, "K": K, "I": I, "E": E, "top": top, "S": S, "S2": S2, "act": act, "residual": residual, "perm": perm,
            "drop": drop, "pad": pad, "out": out}


def listed():
    return [
        # one token into the joint query, key and value projection of an 8B model, which has a bias: latency
        _linear("gemv_1x4096x6144_bias", "gemv", 1, 4096, 6144, S=256, bias=True),
        # sixteen users decoding, down projection of an 8B model, added to the hidden state
        _linear("mx_gemv_16x14336x4096_res", "mx_gemv", 16, 14336, 4096, S=256, residual=True),
        # a short prompt into the gate projection of a 32B model, with its activation
        _linear("mx8_333x5120x27648_silu", "mx8", 333, 5120, 27648, act="silu"),
        # everything at once on rows and features as they come, fp32 output
        _linear("mx8_777x4352x6147_f32", "mx8", 777, 4352, 6147, S=224, bias=True, act="gelu", residual=True, out="f32"),
        # the largest product: down projection of a 70B model over 4096 tokens, added to the hidden state
        _linear("mx8_4096x28672x8192_res", "mx8", 4096, 28672, 8192, residual=True),
        # one token choosing two of eight experts: latency
        _route("route_1x4096_2of8", 1, 4096, 8, 2, renorm=True),
        # 64 tokens choosing eight of 256 experts by sigmoid scores with a bias that balances them
        _route("route_64x8192_8of256", 64, 8192, 256, 8, sigmoid=True, renorm=True, bias=True),
        # one token through eight of 64 small experts: latency
        _moe("mx_moe_1x2048x1024_8of64", "mx_moe", 1, 2048, 1024, 64, 8, residual=True),
        # one token through two of eight experts of an 8B model's width
        _moe("moe_1x4096x14336_2of8", "moe", 1, 4096, 14336, 8, 2, S=256, residual=True),
        # four users, eight of 128 experts each
        _moe("mx_moe_4x4096x1792_8of128", "mx_moe", 4, 4096, 1792, 128, 8),
        # tokens of a padded batch: some choose no expert; odd sizes, channels in the order of the 4-bit path, fp32 hidden state
        _moe("moe_13x5120x1392_4of30_f32", "moe", 13, 5120, 1392, 30, 4, S=208, S2=48, residual=True, perm=True, drop=True, pad=8, out="f32"),
        # the largest: 64 users, every expert busy
        _moe("mx_moe_64x4096x14336_2of8", "mx_moe", 64, 4096, 14336, 8, 2),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["gemv", "mx_gemv", "mx8", "mx8", "route", "moe", "mx_moe", "mx_moe"])
    unit = 16 if op in ("gemv", "moe") else 32
    out = rng.choice(["f16", "f32"])
    pad = rng.choice([0, 0, 8, 64])
    if op == "route":
        E = _log(rng, 2, 512)
        c = _route("", _log(rng, 1, 256), _log(rng, 256, 8192) // 8 * 8, E, min(E, rng.randint(1, 10)), rng.random() < 0.5, rng.random() < 0.7, rng.random() < 0.4, pad)
    elif op in ("moe", "mx_moe"):
        K = _log(rng, 256, 8192) // unit * unit
        I = min(_log(rng, 128, 16384), MOST_EXPERTS // (24 * K)) // unit * unit
        E = max(1, min(_log(rng, 1, 128), MOST_EXPERTS // (3 * K * I)))
        S, S2 = (rng.choice([0, min(n, _log(rng, unit, 1024) // unit * unit)]) for n in (K, I))
        c = _moe("", op, _log(rng, 1, 64), K, I, E, min(E, rng.randint(1, 8)), S, S2, rng.choice(["silu", "silu", *ACTS[1:]]), rng.random() < 0.5,
                 rng.random() < 0.4, rng.random() < 0.3, pad, out)
    else:
        K = max(unit, _log(rng, 256, 28672) // unit * unit)
        N = min(_log(rng, 64, 32768), MOST_WEIGHTS // K)
        if rng.random() < 0.6:
            N = max(16, N // 16 * 16)
        M = _log(rng, 1, 4096) if op == "mx8" else _log(rng, 1, 32)
        M = max(1, min(M, MOST // (K * N)))
        S = rng.choice([0, min(K, _log(rng, unit, 1024) // unit * unit)])
        c = _linear("", op, M, K, N, S, rng.random() < 0.5, rng.choice(ACTS), rng.random() < 0.5, op != "mx8" and rng.random() < 0.4, 0 if op == "mx8" else pad, out)
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------------------------- inputs

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _rows(M, K, pad, factors, gen):
    """fp16 [M, K] inside rows of K + pad: normal values times a factor per channel."""
    buf = torch.zeros((M, K + pad), dtype=torch.float16, device="cuda")
    x = buf[:, :K]
    x.copy_((torch.randn((M, K), device="cuda", generator=gen) * factors).clamp_(-60000.0, 60000.0))
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


def _weights(block, N, K, S, sigma, gen):
    """Packed weights [N, K + S] with the last S channels' blocks twice, N(0, sigma): codes, scale bytes, tensor scale."""
    codes = torch.empty((N, (K + S) // 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty((N, (K + S) // block), dtype=torch.uint8, device="cuda")
    ts = 5.0 * sigma / 2688.0
    step = max(1, (64 << 20) // K)
    for r in range(0, N, step):
        n = min(step, N - r)
        w = torch.randn((n, K // block, block), device="cuda", generator=gen) * sigma
        amax = w.abs().amax(-1)
        if block == 16:
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
    op, M, K = case["op"], case["M"], case["K"]
    s = {"op": op, "case": case, "scratch": torch.empty(SCRATCH, dtype=torch.uint8, device="cuda")}
    if op == "route":
        E = case["E"]
        s["x"] = _rows(M, K, case["pad"], 1.0, gen)
        s["router"] = (torch.randn((E, K), device="cuda", generator=gen) / math.sqrt(K)).half()
        s["bias"] = 0.2 * torch.randn(E, device="cuda", generator=gen) if case["bias"] else None
        s["ids"] = torch.empty((M, case["top"]), dtype=torch.int32, device="cuda")
        s["weights"] = torch.empty((M, case["top"]), dtype=torch.float32, device="cuda")
        return s
    dtype = torch.float32 if case["out"] == "f32" else torch.float16
    factors = _factors(K, gen)
    x = _rows(M, K, case["pad"], factors if op in ("gemv", "mx_gemv", "mx8") else 1.0, gen)
    s["x"] = x
    s["perm"] = torch.randperm(K, device="cuda", generator=gen).int() if case["perm"] else None
    block = 16 if op in ("gemv", "moe") else 32
    N = K if op in ("moe", "mx_moe") else case["N"]
    s["residual"] = torch.randn((M, N), device="cuda", generator=gen).to(dtype) if case["residual"] else None
    s["y"] = torch.empty((M, N), dtype=dtype, device="cuda")
    if op in ("moe", "mx_moe"):
        E, I, top = case["E"], case["I"], case["top"]
        for name, rows, cols, S in (("up", 2 * I, K, case["S"]), ("down", N, I, case["S2"])):
            codes, scales, ts = _weights(block, E * rows, cols, S, 1.0 / math.sqrt(cols), gen)
            s[name + "_codes"], s[name + "_scales"] = codes.reshape(E, rows, -1), scales.reshape(E, rows, -1)
            s[name + "_ts"] = ts * (0.75 + 0.5 * torch.rand(E, device="cuda", generator=gen))
        best = torch.topk(torch.randn((M, E), device="cuda", generator=gen), top)
        s["ids"], s["weights"] = best.indices.int(), torch.softmax(best.values, -1)
        if case["drop"]:
            gone = torch.rand((M, top), device="cuda", generator=gen) < 0.2
            gone[torch.rand(M, device="cuda", generator=gen) < 0.2] = True
            s["ids"] = torch.where(gone, -1, s["ids"])
        return s
    s["w_codes"], s["w_scales"], s["ts"] = _weights(block, N, K, case["S"], 0.02, gen)
    s["bias"] = torch.randn(N, device="cuda", generator=gen).half() if case["bias"] else None
    if op == "mx8":
        s["a_codes"], s["a_scales"] = (t.view(torch.uint8) for t in _mx8(x.float()))
        del s["x"]
    return s


def _mx8(v):
    """fp32 [M, K] -> E4M3 codes [M, K] and E8M0 scales [M, K / 32]."""
    M, K = v.shape
    b = v.reshape(M, K // 32, 32)
    m, e = torch.frexp(b.abs().amax(-1))
    e = torch.where(m > 0, e - 9, 0)
    q = torch.ldexp(b, -e[..., None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    return q.reshape(M, K), (e + 127).to(torch.uint8)


# ------------------------------------------------------------------------------------------------------------ plain forms

def _fp4(codes, scales, K, block):
    """The first K columns of packed weights [..., K + S], in fp32, without the tensor scale."""
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=codes.device)
    c = codes[..., :K // 2].int()
    w = table[torch.stack((c & 15, c >> 4), -1).reshape(*codes.shape[:-1], K // block, block)]
    s = scales[..., :K // block]
    s = s.contiguous().view(torch.float8_e4m3fn).float() if block == 16 else torch.ldexp(torch.ones((), device=s.device), s.int() - 127)
    return (w * s[..., None]).reshape(*codes.shape[:-1], K)


def _act(name, v):
    if name == "relu":
        return torch.where(v < 0, 0.0, v)
    if name == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * v * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v * v * v)))
    if name == "silu":
        return v / (1.0 + torch.exp(-v))
    return v


def _plain_linear(s):
    c = s["case"]
    if s["op"] == "mx8":
        M, K = s["a_codes"].shape
        a = torch.ldexp(s["a_codes"].view(torch.float8_e4m3fn).float().reshape(M, K // 32, 32), s["a_scales"].int()[..., None] - 127).reshape(M, K)
    else:
        K = c["K"]
        a = (s["x"] if s["perm"] is None else s["x"][:, s["perm"]]).float()
    y = a @ _fp4(s["w_codes"], s["w_scales"], K, 16 if s["op"] == "gemv" else 32).T
    if s["op"] == "gemv":
        y = y * s["ts"]
    if s["bias"] is not None:
        y = y + s["bias"].float()
    y = _act(c["act"], y)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["y"].dtype)


def _plain_route(s):
    c = s["case"]
    logits = s["x"].double() @ s["router"].double().T
    if c["sigmoid"]:
        score = 1.0 / (1.0 + torch.exp(-logits))
        rank = logits if s["bias"] is None else score + s["bias"].double()
    else:
        score = torch.exp(logits - logits.amax(-1, keepdim=True))
        score = score / score.sum(-1, keepdim=True)
        rank = logits if s["bias"] is None else score + s["bias"].double()
    ids = torch.sort(rank, dim=-1, descending=True, stable=True).indices[:, :c["top"]]
    w = torch.gather(score, 1, ids)
    if c["renorm"]:
        w = w / w.sum(-1, keepdim=True)
    return ids.int(), w.float()


def _plain_experts(s):
    """Every expert for every token where there are no more experts than choices; the chosen ones otherwise."""
    c, ids, w = s["case"], s["ids"], s["weights"]
    M, K, I, E, top = (c[k] for k in ("M", "K", "I", "E", "top"))
    block = 16 if s["op"] == "moe" else 32
    x = (s["x"] if s["perm"] is None else s["x"][:, s["perm"]]).float()
    if E <= M * top:
        which = torch.arange(E, device="cuda")
        share = (w[:, :, None] * (ids[:, :, None] == which)).sum(1)
    else:
        which = ids.reshape(-1).clamp(min=0).long()
        share = torch.where(ids < 0, 0.0, w).reshape(1, -1) * (torch.arange(M * top, device="cuda") // top == torch.arange(M, device="cuda")[:, None])
    y = torch.zeros((M, K), device="cuda")
    step = max(1, (1 << 30) // (3 * K * I))         # experts at a time: their weights in 32 bits fill 4 GiB
    for at in range(0, which.numel(), step):
        e, part = which[at:at + step], share[:, at:at + step]
        v = x @ _fp4(s["up_codes"][e], s["up_scales"][e], K, block).reshape(-1, K).T
        v = v.reshape(M, -1, 2, I)
        d = _fp4(s["down_codes"][e], s["down_scales"][e], I, block)
        if block == 16:
            v = v * s["up_ts"][e][:, None, None]
            d = d * s["down_ts"][e][:, None, None]
        h = _act(c["act"], v[:, :, 0]) * v[:, :, 1] * part[:, :, None]
        y = y + h.reshape(M, -1) @ d.transpose(0, 1).reshape(K, -1).T
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["y"].dtype)


def _library(s):
    from paper_2601_07475_amd import binding as B
    c, op = s["case"], s["op"]
    if op == "route":
        flags = (B.MOE_SIGMOID if c["sigmoid"] else 0) | (B.MOE_RENORMALIZE if c["renorm"] else 0)
        return B.arcq_moe_route(s["x"], s["router"], c["top"], bias=s["bias"], flags=flags, ids=s["ids"], weights=s["weights"], workspace=s["scratch"])
    act = {"none": B.ACT_NONE, "relu": B.ACT_RELU, "gelu": B.ACT_GELU, "gelu_tanh": B.ACT_GELU_TANH, "silu": B.ACT_SILU}[c["act"]]
    end = {"activation": act, "residual": s["residual"], "y": s["y"], "workspace": s["scratch"]}
    if op == "gemv":
        return B.arcq_gemv_epilogue(s["x"], s["perm"], s["w_codes"], s["w_scales"], s["ts"], bias=s["bias"], **end)
    if op == "mx_gemv":
        return B.arcq_mx_gemv_epilogue(s["x"], s["perm"], s["w_codes"], s["w_scales"], bias=s["bias"], **end)
    if op == "mx8":
        return B.arcq_mx8_gemm_epilogue(s["a_codes"], s["a_scales"], s["w_codes"], s["w_scales"], bias=s["bias"], **end)
    if op == "moe":
        return B.arcq_moe(s["x"], s["perm"], s["ids"], s["weights"], s["up_codes"], s["up_scales"], s["up_ts"], s["down_codes"], s["down_scales"],
                          s["down_ts"], **end)
    return B.arcq_mx_moe(s["x"], s["perm"], s["ids"], s["weights"], s["up_codes"], s["up_scales"], s["down_codes"], s["down_scales"], **end)


def run(state):
    if own:
        return _library(state)
    return _plain_route(state) if state["op"] == "route" else _plain_experts(state) if state["op"] in ("moe", "mx_moe") else _plain_linear(state)


def work(case):
    op, M, K = case["op"], case["M"], case["K"]
    if op == "route":
        E, top = case["E"], case["top"]
        return {"bytes": 2 * M * K + 2 * E * K + (4 * E if case["bias"] else 0) + 8 * M * top, "flops": 2 * M * K * E}
    size = 4 if case["out"] == "f32" else 2
    per = 9 / 16 if op in ("gemv", "moe") else 17 / 32           # bytes of a packed weight with its share of the scale
    order = 4 * K if case["perm"] else 0
    if op in ("moe", "mx_moe"):
        I, E, top = case["I"], case["E"], case["top"]
        live = M * top * (0.64 if case["drop"] else 1.0)
        used = E * (1.0 - (1.0 - top / E) ** (live / top))       # experts that some token chooses, on average
        return {"bytes": int(used * 3 * K * I * per) + 2 * M * K + order + 8 * M * top + M * K * size * (2 if case["residual"] else 1), "flops": int(6 * live * K * I)}
    N = case["N"]
    a = M * K + M * K // 32 if op == "mx8" else 2 * M * K + order
    return {"bytes": int(N * K * per) + a + M * N * size * (2 if case["residual"] else 1) + (2 * N if case["bias"] else 0), "flops": 2 * M * N * K}


# ------------------------------------------------------------------------------------------------ definitions, in 64 bits

def _exact_weights(codes, scales, K, block):
    """fp64 [rows, K] of packed rows, without the tensor scale."""
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


def _exact_act(name, v):
    if name == "relu":
        return v.clamp(min=0.0)
    if name == "gelu":
        return v * torch.special.erfc(-v / math.sqrt(2.0)) / 2.0
    if name == "gelu_tanh":
        return v * torch.sigmoid(math.sqrt(8.0 / math.pi) * (v + 0.044715 * v ** 3))        # (1 + tanh u) / 2 = sigmoid(2 u)
    if name == "silu":
        return v * torch.sigmoid(v)
    return v


def exact(case, seed):
    s = prepare(case, seed)
    op, K = case["op"], case["K"]
    if op == "route":
        x, r = s["x"].double(), s["router"].double()
        logits = torch.stack([x @ row for row in r], 1)
        score = torch.sigmoid(logits) if case["sigmoid"] else torch.softmax(logits, 1)
        rank = score if s["bias"] is None else score + s["bias"].double()
        chosen = []
        left = rank.clone()
        for _ in range(case["top"]):
            best = (left == left.amax(1, keepdim=True)).int().argmax(1)
            chosen.append(best)
            left.scatter_(1, best[:, None], -math.inf)
        ids = torch.stack(chosen, 1)
        w = score.gather(1, ids)
        return ids.int(), w / w.sum(1, keepdim=True) if case["renorm"] else w
    block = 16 if op in ("gemv", "moe") else 32
    if op == "mx8":
        a = s["a_codes"].view(torch.float8_e4m3fn).double().reshape(-1, K // 32, 32)
        a = (a * torch.exp2(s["a_scales"].double() - 127)[..., None]).reshape(-1, K)
    else:
        a = s["x"].double() if s["perm"] is None else s["x"].double()[:, s["perm"].long()]
    if op in ("moe", "mx_moe"):
        I = case["I"]
        y = torch.zeros((case["M"], K), dtype=torch.float64, device="cuda")
        for e in range(case["E"]):
            m, j = torch.nonzero(s["ids"] == e, as_tuple=True)
            if m.numel() == 0:
                continue
            up = a[m] @ _exact_weights(s["up_codes"][e], s["up_scales"][e], K, block).T
            down = _exact_weights(s["down_codes"][e], s["down_scales"][e], I, block)
            if block == 16:
                up, down = up * s["up_ts"][e].double(), down * s["down_ts"][e].double()
            y.index_add_(0, m, s["weights"][m, j].double()[:, None] * ((_exact_act(case["act"], up[:, :I]) * up[:, I:]) @ down.T))
    else:
        y = a @ _exact_weights(s["w_codes"], s["w_scales"], K, block).T * (s["ts"] if op == "gemv" else 1.0)
        if s["bias"] is not None:
            y = y + s["bias"].double()
        y = _exact_act(case["act"], y)
    return y if s["residual"] is None else y + s["residual"].double()
