"""The operators around and inside a linear layer whose weights are held in 4 bits, as cases that can be timed and compared.

What a serving program does per layer and per answer: the residual is added and the sum normalised, the result is handed
to the next product in 16 bits, or in 8 or 4 bits with one scale for each 32 channels (microscaled, MX); the product multiplies it with weights held in
MX 4-bit form; behind the last product the log probabilities of given tokens, the entropy and the most
probable alternatives are taken from the logits.  Offline (and for activations online) values are brought into the MX forms and read back.

Formulas.  MX: for every 32 consecutive channels of a row, e = max(floor(log2(largest magnitude)) - emax, -127), the scale is
2^e, an element is its value / 2^e rounded to the nearest number of its format, ties to even, no further than the largest one:
4 bits: 0 0.5 1 1.5 2 3 4 6 and their negatives (emax 2); 8 bits: 1 sign, 4 exponent and 3 mantissa bits, up to 448 (emax 8).  A
row is padded with zeros to a multiple of 128 channels; 4-bit elements stand two to a byte, the even channel in the low half; a scale is one byte, e + 127,
and the four scales of a row's 128 channels stand behind those of the row before it: [128 channels][row][4].
Norm: h = x + r rounded to the type of x; y = h w / sqrt(mean(h^2) + eps).  Product: Y = X W^T.  Log probabilities: log softmax.

Shapes are those of the workloads in workloads.py and generic ones, ragged ones beside them; weights are N(0, K^-1/2), activations
normal with a log-normal scale per channel and a few outlier channels, logits normal with a wide scale.
"""
import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
#: smallest exponent of a normal element, mantissa bits, largest element, exponent of the largest element
FORMATS = {"fp4": (0, 1, 6.0, 2), "fp8": (-6, 3, 448.0, 8)}


# ---- the cases ------------------------------------------------------------------------------------
def listed():
    return [
        # a short prompt's activations to 8 bits with scales and back, sizes that are no multiple of anything
        dict(name="quantise_ragged", kind="quantise", R=333, K=5003, fmt="fp8", dtype="bf16"),
        # the gate matrix of a 7B layer to 4 bits and back
        dict(name="quantise_weights", kind="quantise", R=11008, K=4096, fmt="fp4", dtype="f16"),
        # smallest call: the norm in front of a layer while one sequence is decoded
        dict(name="norm_token", kind="norm", R=1, K=4096, out="16", dtype="bf16"),
        # the norm in front of a layer on a prompt, its output in 8 bits with scales for the product
        dict(name="norm_prompt", kind="norm", R=2048, K=8192, out="fp8", dtype="f16"),
        # decoding one sequence: gate matrix of a 7B layer, activations in 16 bits
        dict(name="product_token", kind="product", M=1, N=11008, K=4096, act="16", dtype="f16"),
        # decoding sixteen sequences: gate matrix of a 65B layer, activations in 8 bits
        dict(name="product_decode", kind="product", M=16, N=22016, K=8192, act="fp8", dtype="bf16"),
        # a short prompt through a layer whose sizes are no multiple of any tile, activations in 16 bits
        dict(name="product_ragged", kind="product", M=333, N=5003, K=3020, act="16", dtype="bf16"),
        # a long prompt through the gate matrix of a 13B layer, activations in 8 bits
        dict(name="product_prefill_8", kind="product", M=2048, N=13824, K=5120, act="fp8", dtype="f16"),
        # a long prompt through the gate matrix of a 65B layer, activations in 4 bits as well
        dict(name="product_prefill_4", kind="product", M=2048, N=22016, K=8192, act="fp4", dtype="bf16"),
        # decoding: the answers of eight sequences, with twenty alternatives each
        dict(name="logprobs_decode", kind="logprobs", R=8, V=131072, top=20, dtype="bf16"),
        # perplexity of a prompt: the log probabilities and entropies of its tokens, no alternatives
        dict(name="logprobs_prompt", kind="logprobs", R=2048, V=32000, top=0, dtype="f16"),
        # a prompt scored with 32-bit logits, an odd vocabulary, and five alternatives each
        dict(name="logprobs_ragged", kind="logprobs", R=555, V=50021, top=5, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Half the time a multiple of 256, else anything."""
    v = _log_int(rng, lo, hi)
    return v if rng.random() < 0.5 else max(256, v // 256 * 256)


def draw(rng):
    kind = rng.choice(["quantise", "norm", "product", "product", "product", "logprobs"])
    dtype = rng.choice(["f16", "bf16"])
    if kind == "quantise":
        return dict(kind=kind, R=_log_int(rng, 1, 11008), K=_size(rng, 64, 13824), fmt=rng.choice(["fp4", "fp8"]), dtype=dtype)
    if kind == "norm":
        return dict(kind=kind, R=_log_int(rng, 1, 4096), K=_size(rng, 64, 16384), out=rng.choice(["16", "fp8", "fp8", "fp4"]), dtype=dtype)
    if kind == "product":
        M, N, K = _log_int(rng, 1, 2048), _size(rng, 256, 22016), _size(rng, 256, 13824)
        while M * N * K > 2048 * 22016 * 8192:
            N = max(256, N // 2)
        return dict(kind=kind, M=M, N=N, K=K, act=rng.choice(["16", "fp8", "fp4"]), dtype=dtype)
    return dict(kind=kind, R=_log_int(rng, 1, 2048), V=_size(rng, 1000, 131072), top=rng.choice([0, 1, 5, 20]), dtype=rng.choice(["f16", "bf16", "f32"]))


# ---- inputs ---------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _features(g, T, K, dtype):
    s = torch.exp(torch.randn(K, device="cuda", generator=g))
    few = torch.randperm(K, device="cuda", generator=g)[: max(1, round(0.005 * K))]
    s[few] *= 30.0
    return (torch.randn(T, K, device="cuda", generator=g) * s).clamp_(-60000, 60000).to(dtype)


def _weights(g, N, K, dtype):
    return (torch.randn(N, K, device="cuda", generator=g) * K ** -0.5).to(dtype)


def _inputs(case, seed):
    """The user's tensors in 16 or 32 bits, from the seed alone."""
    g, dt, kind = _gen(seed), DTYPES[case["dtype"]], case["kind"]
    if kind == "quantise":
        x = _weights(g, case["R"], case["K"], dt) if case["fmt"] == "fp4" else _features(g, case["R"], case["K"], dt)
        return dict(x=x)
    if kind == "norm":
        x = _features(g, case["R"], case["K"], dt)
        r = _features(g, case["R"], case["K"], dt)
        w = (1.0 + 0.2 * torch.randn(case["K"], device="cuda", generator=g)).to(dt)
        return dict(x=x, residual=r, weight=w, eps=1e-5)
    if kind == "product":
        return dict(x=_features(g, case["M"], case["K"], dt), w=_weights(g, case["N"], case["K"], dt))
    logits = (torch.randn(case["R"], case["V"], device="cuda", generator=g) * 3.0).to(dt)
    tokens = torch.randint(0, case["V"], (case["R"],), device="cuda", generator=g)
    return dict(logits=logits, tokens=tokens)


# ---- the plain forms, in 32 bits ------------------------------------------------------------------
def _blocks(x):
    """x[R, K] in 32 bits, padded to a multiple of 128 channels and cut into blocks of 32."""
    x = torch.nn.functional.pad(x.float(), (0, -x.shape[1] % 128))
    return x.reshape(x.shape[0], -1, 32)


def _scale_exponents(b, fmt):
    amax = b.abs().amax(2)
    e = torch.frexp(amax)[1] - 1 - FORMATS[fmt][3]
    return torch.where(amax == 0, -127, e).clamp_(min=-127)


def _elements(b, e, fmt):
    """The numbers of the format nearest to b / 2^e."""
    low, bits, most, _ = FORMATS[fmt]
    y = b * torch.exp2(-e.float())[:, :, None]
    step = torch.exp2((torch.frexp(y)[1] - 1).clamp_(min=low).float() - bits)
    return (torch.round(y / step) * step).clamp_(-most, most)


def _quantised(x, fmt):
    """(elements [R, Kp/32, 32] as 32-bit numbers, exponents [R, Kp/32])"""
    b = _blocks(x)
    e = _scale_exponents(b, fmt)
    return _elements(b, e, fmt), e


def _encoded(x, fmt):
    """MX form of x: element codes [R, bytes] and scales [Kp/128, R, 4], one byte each."""
    data, scales = [], []
    rows = max(1, (1 << 25) // max(1, x.shape[1]))
    for lo in range(0, x.shape[0], rows):
        v, e = _quantised(x[lo:lo + rows], fmt)
        if fmt == "fp8":
            data.append(v.to(torch.float8_e4m3fn).view(torch.uint8).reshape(v.shape[0], -1))
        else:
            a = v.abs()
            code = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, 4 + a / 2)).to(torch.uint8)
            code += (v < 0).to(torch.uint8) * 8
            code = code.reshape(v.shape[0], -1, 2)
            data.append(code[:, :, 0] | code[:, :, 1] << 4)
        scales.append((e + 127).to(torch.uint8).reshape(e.shape[0], -1, 4).transpose(0, 1))
    return torch.cat(data), torch.cat(scales, 1).contiguous()


def _decoded(data, scales, fmt):
    """The numbers [R, Kp] in 32 bits that an MX form stands for."""
    if fmt == "fp8":
        v = data.view(torch.float8_e4m3fn).float()
    else:
        table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=data.device)
        v = table[torch.stack((data & 15, data >> 4), 2).int()].reshape(data.shape[0], -1)
    s = torch.exp2(scales.transpose(0, 1).reshape(data.shape[0], -1).float() - 127.0)
    return (v.reshape(v.shape[0], -1, 32) * s[:, :, None]).reshape(v.shape[0], -1)


def _round_trip(x, fmt, dtype):
    v, e = _quantised(x, fmt)
    return (v * torch.exp2(e.float())[:, :, None]).reshape(x.shape[0], -1)[:, : x.shape[1]].to(dtype)


def _plain(s):
    kind = s["kind"]
    if kind == "quantise":
        return dict(values=_round_trip(s["x"], s["fmt"], s["x"].dtype))
    if kind == "norm":
        x = s["x"]
        h = (x.float() + s["residual"].float()).to(x.dtype)
        f = h.float()
        y = f * torch.rsqrt(f.square().mean(1, keepdim=True) + s["eps"]) * s["weight"].float()
        return dict(residual=h, y=y.to(x.dtype) if s["out"] == "16" else _round_trip(y, s["out"], x.dtype))
    if kind == "product":
        w = _decoded(s["w_data"], s["w_scales"], "fp4")[:, : s["K"]]
        if s["act"] == "16":
            x = s["x"].float()
        else:
            x = _decoded(s["x_data"], s["x_scales"], s["act"])[:, : s["K"]]
        return dict(y=(x @ w.t()).to(s["dtype"]))
    x = s["logits"].float()
    m = x.amax(1, keepdim=True)
    p = torch.exp(x - m)
    z = p.sum(1, keepdim=True)
    lse = m + torch.log(z)
    out = dict(logprob=(x.gather(1, s["tokens"][:, None]) - lse)[:, 0],
               entropy=(torch.log(z) - (p * (x - m)).sum(1, keepdim=True) / z)[:, 0])
    if s["top"]:
        value, ids = torch.sort(x, dim=1, descending=True, stable=True)
        out.update(top_ids=ids[:, : s["top"]].int(), top_logprobs=value[:, : s["top"]] - lse)
    return out


# ---- what a program holds, and one pass -----------------------------------------------------------
def prepare(case, seed):
    state = dict(case)
    state.update(_inputs(case, seed))
    state["dtype"] = DTYPES[case["dtype"]]
    if case["kind"] == "product":
        state["w_data"], state["w_scales"] = _encoded(state.pop("w"), "fp4")
        if case["act"] != "16":
            state["x_data"], state["x_scales"] = _encoded(state.pop("x"), case["act"])
    if own:
        import paper_2310_15929_amd as esp
        state["ctx"] = ctx = esp.Context(0)
        state["formats"] = {"fp4": esp.MX_FP4, "fp8": esp.MX_FP8, "16": None}
        if case["kind"] == "product":
            state["w"] = ctx.mx_pack(esp.MX(state["w_data"], state["w_scales"], case["K"], esp.MX_FP4))
            if case["act"] != "16":
                state["x"] = esp.MX(state["x_data"], state["x_scales"], case["K"], state["formats"][case["act"]])
    return state


def run(state):
    if not own:
        return _plain(state)
    ctx, kind = state["ctx"], state["kind"]
    if kind == "quantise":
        q = ctx.mx_quantize(state["x"], state["formats"][state["fmt"]])
        return dict(values=ctx.mx_dequantize(q, state["dtype"]))
    if kind == "norm":
        y, h = ctx.rms_norm(state["x"], state["weight"], state["eps"], residual=state["residual"], fmt=state["formats"][state["out"]])
        return dict(residual=h, y=y if state["out"] == "16" else ctx.mx_dequantize(y, state["dtype"]))
    if kind == "product":
        return dict(y=ctx.mx_gemm(state["x"], state["w"], dtype=state["dtype"]))
    r = ctx.token_logprobs(state["logits"], state["tokens"], top=state["top"])
    out = dict(logprob=r.logprob, entropy=r.entropy)
    if state["top"]:
        out.update(top_ids=r.top_ids, top_logprobs=r.top_logprobs)
    return out


# ---- what a pass cannot do without ----------------------------------------------------------------
def _held(R, K, fmt):
    """Bytes of R x K numbers in a format."""
    return 2 * R * K if fmt == "16" else R * K * (16 if fmt == "fp4" else 32) // 32 + R * -(-K // 32)


def work(case):
    kind = case["kind"]
    if kind == "quantise":
        # values read, the MX form written and read back, values written
        n = case["R"] * case["K"]
        return {"bytes": 4 * n + 2 * _held(case["R"], case["K"], case["fmt"]), "flops": 4 * n}
    if kind == "norm":
        # both inputs read, sum and output written; an output in fewer bits is read back into 16
        n = case["R"] * case["K"]
        back = 0 if case["out"] == "16" else _held(case["R"], case["K"], case["out"]) + 2 * n
        return {"bytes": 6 * n + 2 * case["K"] + _held(case["R"], case["K"], case["out"]) + back, "flops": 5 * n}
    if kind == "product":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": _held(N, K, "fp4") + _held(M, K, case["act"]) + 2 * M * N, "flops": 2 * M * N * K}
    n = case["R"] * case["V"]
    return {"bytes": n * (4 if case["dtype"] == "f32" else 2) + case["R"] * (16 + 8 * case["top"]), "flops": 6 * n}


# ---- the same in 64 bits, from the definitions ----------------------------------------------------
def _nearest(values, fmt, dtype=torch.float64):
    """MX round trip in 64 bits by looking the two neighbours up in the list of the format's numbers."""
    R, K = values.shape
    if fmt == "fp4":
        grid = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    else:
        grid = [k * 2.0 ** -9 for k in range(8)] + [(8 + k) * 2.0 ** (p - 3) for p in range(-6, 9) for k in range(8)][:-1]
    grid = torch.tensor(grid, dtype=torch.float64, device=values.device)
    out = torch.zeros(R, -(-K // 32) * 32, dtype=torch.float64, device=values.device)
    rows = max(1, (1 << 24) // max(1, K))
    for lo in range(0, R, rows):
        v = torch.zeros(min(rows, R - lo), out.shape[1], dtype=torch.float64, device=values.device)
        v[:, :K] = values[lo:lo + rows]
        v = v.reshape(v.shape[0], -1, 32)
        top = v.abs().max(dim=2, keepdim=True).values
        e = torch.log2(top.clamp_min(2.0 ** -200)).floor()
        e = e - (top < torch.exp2(e)).double() + (top >= torch.exp2(e + 1)).double()  # where the logarithm was rounded across
        scale = torch.exp2((e - FORMATS[fmt][3]).clamp_min(-127))
        a = v.abs() / scale
        hi = torch.searchsorted(grid, a).clamp_(max=len(grid) - 1)
        below = (hi - 1).clamp_(min=0)
        up, down = grid[hi] - a, a - grid[below]
        pick = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, below)
        out[lo:lo + rows] = (torch.copysign(grid[pick], v) * scale).reshape(v.shape[0], -1)
    return out[:, :K].to(dtype)


def exact(case, seed):
    kind = case["kind"]
    s = _inputs(case, seed)
    if kind == "quantise":
        return dict(values=_nearest(s["x"].double(), case["fmt"]))
    if kind == "norm":
        h = (s["x"].double() + s["residual"].double()).to(s["x"].dtype).double()
        y = h * s["weight"].double() / torch.sqrt((h * h).sum(1, keepdim=True) / case["K"] + s["eps"])
        return dict(residual=h, y=y if case["out"] == "16" else _nearest(y, case["out"]))
    if kind == "product":
        w = _nearest(s["w"].double(), "fp4")
        x = s["x"].double() if case["act"] == "16" else _nearest(s["x"].double(), case["act"])
        return dict(y=x @ w.t())
    lp = torch.log_softmax(s["logits"].double(), 1)
    out = dict(logprob=lp[torch.arange(case["R"], device=lp.device), s["tokens"]], entropy=-(lp.exp() * lp).sum(1))
    if case["top"]:
        out.update(top_ids=None, top_logprobs=torch.topk(lp, case["top"], dim=1).values)
    return out
