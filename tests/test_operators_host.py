"""The operators around a 4-bit linear layer without a GPU: pins of the oracle, size queries, refusals."""
import ctypes as C
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

import paper_2310_15929_amd as esp
from oracle import operators_oracle as orc

EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -7
P = 4096        # stands for a device pointer: aligned, never followed


@pytest.fixture(scope="module")
def ctx():
    return esp.Context(0)


# ---- oracle ---------------------------------------------------------------------------------------
def test_fp8_codes_are_those_of_torch():
    v = orc.mx_values(np.arange(256, dtype=np.uint8)[None, :], np.full((1, 8), 127, np.uint8), orc.FP8)[0]
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(v, want, equal_nan=True)


def test_worked_block():
    x = np.zeros((1, 32))
    x[0, :8] = [7.0, 5.0, -2.5, 0.25, 0.75, 0.2, -0.3, 3.5]   # largest 7: scale 1; ties to even, 7 and more to 6
    code, E = orc.mx_quantize(x, orc.FP4)
    assert E[0, 0] == 127
    assert list(orc.mx_values(code, E, orc.FP4)[0, :8]) == [6.0, 4.0, -2.0, 0.0, 1.0, 0.0, -0.5, 4.0]
    code, E = orc.mx_quantize(x, orc.FP8)   # scale 2^(2 - 8)
    assert E[0, 0] == 121 and list(orc.mx_values(code, E, orc.FP8)[0, :4]) == [7.0, 5.0, -2.5, 0.25]


@pytest.mark.parametrize("fmt", [orc.FP4, orc.FP8])
def test_error_is_half_a_step_or_the_limit(fmt):
    x = np.random.default_rng(1).standard_normal((40, 128))
    code, E = orc.mx_quantize(x, fmt)
    v = orc.mx_values(code, E, fmt)
    s = np.repeat(np.ldexp(1.0, E.astype(int) - 127), 32, 1)
    a = np.abs(x) / s
    most = orc.GRID[fmt][-1]
    inside = a <= most
    half = 2.0 ** -2 if fmt == orc.FP4 else 2.0 ** -4   # of a value: one or three bits behind the first
    assert (np.abs(v - x)[inside] <= np.maximum(half * np.abs(x), s * orc.GRID[fmt][1] / 2)[inside]).all()
    assert (np.abs(v)[~inside] == (most * s)[~inside]).all()


def test_log_probabilities_of_a_uniform_row():
    lp, ent, ids, tops = orc.token_logprobs(np.zeros((1, 8)), [3], 2)
    assert math.isclose(lp[0], -math.log(8)) and math.isclose(ent[0], math.log(8)) and list(ids[0]) == [0, 1] and math.isclose(tops[0, 1], -math.log(8))


# ---- sizes ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("R,K", [(0, 1), (1, 1), (3, 127), (5, 128), (7, 5003)])
def test_sizes(R, K):
    kp = -(-K // 128) * 128
    assert esp.mx_size(R, K, esp.MX_FP4) == (R * kp // 2, R * kp // 32)
    assert esp.mx_size(R, K, esp.MX_FP8) == (R * kp, R * kp // 32)
    if R:
        assert esp.mx_packed_size(R, K) == -(-R // 64) * 64 * kp * 17 // 32
    assert esp.mx_gemm_workspace(0, 64, K, 2) == 0
    assert esp.token_logprobs_workspace(0, K, esp.F32, 1) == 0


@pytest.mark.parametrize("call", [
    lambda: esp.mx_size(-1, 8, 0), lambda: esp.mx_size(1, 0, 0), lambda: esp.mx_size(1 << 22, 8, 0), lambda: esp.mx_size(1, 8, 2),
    lambda: esp.mx_size(1 << 21, 1 << 20, 0), lambda: esp.mx_packed_size(0, 8), lambda: esp.mx_packed_size(8, 0),
    lambda: esp.mx_gemm_workspace(-1, 8, 8, 0), lambda: esp.mx_gemm_workspace(1, 8, 8, 3), lambda: esp.mx_gemm_workspace(1, 0, 8, 0),
    lambda: esp.token_logprobs_workspace(1, 8, 3, 0), lambda: esp.token_logprobs_workspace(1, 8, 0, 9),
    lambda: esp.token_logprobs_workspace(1, 100, 0, 33), lambda: esp.token_logprobs_workspace(1, (1 << 21) + 1, 0, 0)])
def test_size_queries_refuse(call):
    with pytest.raises(esp.EsparseError):
        call()


# ---- the choice of a kernel of the product ----------------------------------------------------------
@pytest.fixture(scope="module")
def choice():
    spec = importlib.util.spec_from_file_location("mx_kernel_choice", os.path.join(os.path.dirname(__file__), "..", "profiles", "mx_kernel_choice.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("act", ["fp8", "fp4", "16"])
def test_choice_is_near_the_fastest_kernel(choice, act):
    """What the source says of its tables, from the times beside them."""
    source, cases = open(choice.SOURCE).read(), choice.read_times()[act]
    kernels = {**choice.table(source, "rows", act), **choice.table(source, "tile", act)}
    assert len(kernels) == 15 and len(cases) == 234
    ratios = [cells[choice.choose(kernels, *product)] / min(cells.values()) for product, cells in cases.items()]
    assert np.mean(ratios) <= 1.0115 and max(ratios) <= 1.23


def test_sizes_of_the_gpu_tests_reach_every_kernel(choice):
    """The sizes of test_operators_gpu.KERNEL_SIZES, in the order of the tables."""
    from test_operators_gpu import KERNEL_SIZES
    source = open(choice.SOURCE).read()
    for act, sizes in KERNEL_SIZES.items():
        kernels = {**choice.table(source, "rows", act), **choice.table(source, "tile", act)}
        assert [choice.choose(kernels, *size)[0] for size in sizes] == list(kernels), act


# ---- refusals of the C calls (before any device call) -----------------------------------------------
def _expect(ctx, rc, code, word):
    assert rc == code
    assert word.encode() in ctx._lib.esparse_last_error(ctx._h), ctx._lib.esparse_last_error(ctx._h)


@pytest.mark.parametrize("args,code,word", [
    ((P, 2, 8, 8, 5, 0, P, P), EUNSUPPORTED, "dtype"), ((P, 2, 8, 8, 0, 2, P, P), EUNSUPPORTED, "format"), ((None, 2, 8, 8, 0, 0, P, P), EINVAL, "null"),
    ((P, 2, 8, 8, 0, 0, None, P), EINVAL, "null"), ((P, 2, 8, 8, 0, 0, P, None), EINVAL, "null"), ((P, 2, 8, 7, 0, 0, P, P), EINVAL, "ldx"),
    ((P, -1, 8, 8, 0, 0, P, P), EINVAL, "rows"), ((P, 1 << 22, 8, 8, 0, 0, P, P), EINVAL, "rows"), ((P, 2, 0, 8, 0, 0, P, P), EINVAL, "range"),
    ((P + 1, 2, 8, 8, 0, 0, P, P), EINVAL, "aligned"), ((P + 2, 2, 8, 8, 2, 0, P, P), EINVAL, "aligned"), ((P, 2, 8, 8, 0, 0, P + 8, P), EINVAL, "16-byte"),
    ((P, 1 << 21, 1 << 20, 1 << 20, 0, 0, P, P), EINVAL, "2^34"),
    ((P, 2, 8, 8, 0, 0, P, P << 4), EINVAL, "overlaps"), ((P, 2, 8, 8, 0, 0, P << 4, P), EINVAL, "overlaps"), ((P, 2, 8, 8, 0, 0, P << 4, (P << 4) + 64), EINVAL, "overlaps"),
    ((P, 9, 8, 800, 2, 1, P + 20000, P << 4), EINVAL, "overlaps")])
def test_quantize_refuses(ctx, args, code, word):
    _expect(ctx, ctx._lib.esparse_mx_quantize(ctx._h, *args), code, word)


@pytest.mark.parametrize("args,code,word", [
    ((P, P, 2, 8, 0, 4, P), EUNSUPPORTED, "dtype"), ((P, P, 2, 8, 3, 0, P), EUNSUPPORTED, "format"), ((None, P, 2, 8, 0, 0, P), EINVAL, "null"),
    ((P, P, 2, 8, 0, 0, None), EINVAL, "null"), ((P, P + 4, 2, 8, 0, 0, P), EINVAL, "16-byte"), ((P, P, 2, 8, 0, 2, P + 2), EINVAL, "aligned"), ((P, P << 4, 2, 8, 0, 0, P + 16), EINVAL, "overlaps"),
    ((P << 4, P, 2, 8, 0, 0, P), EINVAL, "overlaps")])
def test_dequantize_refuses(ctx, args, code, word):
    _expect(ctx, ctx._lib.esparse_mx_dequantize(ctx._h, *args), code, word)


@pytest.mark.parametrize("args,code,word", [((None, P, 2, 8, P), EINVAL, "null"), ((P, P, 0, 8, P), EINVAL, "N"), ((P, P, 2, 8, P + 8), EINVAL, "16-byte"),
                                            ((P, P << 4, 2, 8, P), EINVAL, "overlaps"), ((P << 4, P, 200, 8, P - 64), EINVAL, "overlaps")])
def test_pack_refuses(ctx, args, code, word):
    _expect(ctx, ctx._lib.esparse_mx_pack(ctx._h, *args), code, word)


#         X, scales, M, ldx, act, dtype, w, N, K, out, Y, ws, bytes
GEMM = dict(X=P, xs=P << 4, M=4, ldx=0, act=1, dtype=0, w=P << 5, N=64, K=128, out=1, Y=P << 8, ws=None, nbytes=0)


@pytest.mark.parametrize("change,code,word", [
    (dict(out=3), EUNSUPPORTED, "dtype"), (dict(act=3), EUNSUPPORTED, "act"), (dict(act=2, dtype=2, ldx=128), EUNSUPPORTED, "dtype"), (dict(M=-1), EINVAL, "range"),
    (dict(N=0), EINVAL, "range"), (dict(K=0), EINVAL, "range"), (dict(X=None), EINVAL, "null"), (dict(w=None), EINVAL, "null"), (dict(Y=None), EINVAL, "null"),
    (dict(xs=None), EINVAL, "x_scales"), (dict(X=P + 8), EINVAL, "16-byte"), (dict(w=P + 8), EINVAL, "16-byte"), (dict(Y=P + 8), EINVAL, "16-byte"),
    (dict(act=2, ldx=127), EINVAL, "ldx"), (dict(act=2, ldx=128, X=P + 1), EINVAL, "aligned"), (dict(act=2, ldx=128, K=127), EINVAL, "workspace"),
    (dict(act=2, ldx=128, K=127, ws=P, nbytes=8), EWORKSPACE, "workspace"), (dict(act=2, ldx=128, K=127, ws=(P << 9) + 16, nbytes=1 << 30), EINVAL, "256-byte"),
    (dict(act=2, ldx=129), EINVAL, "workspace"), (dict(act=2, ldx=128, X=P + 8), EINVAL, "workspace"), (dict(act=2, ldx=(1 << 22) + 8), EINVAL, "ldx"),
    (dict(K=(1 << 22) + 1), EINVAL, "range"), (dict(Y=P), EINVAL, "overlaps"), (dict(Y=P << 4), EINVAL, "overlaps"),
    (dict(Y=(P << 5) + 4096), EINVAL, "overlaps"), (dict(act=2, ldx=127, K=127, ws=P << 8, nbytes=1 << 30), EINVAL, "overlaps"),
    (dict(act=2, ldx=127, K=127, ws=P, nbytes=1 << 30), EINVAL, "overlaps")])
def test_gemm_refuses(ctx, change, code, word):
    a = {**GEMM, **change}
    _expect(ctx, ctx._lib.esparse_mx_gemm(ctx._h, a["X"], a["xs"], a["M"], a["ldx"], a["act"], a["dtype"], a["w"], a["N"], a["K"], a["out"], a["Y"], a["ws"],
                                          a["nbytes"]), code, word)


def test_gemm_ignores_scales_of_16_bit_activations(ctx):
    """x_scales inside Y or the workspace: no overlap with activations that have none (the call gets as far as the missing workspace)."""
    for change in (dict(xs=(P << 8) + 64), dict(xs=(P << 9) + 64, ws=P << 9, nbytes=8)):
        a = {**GEMM, "act": 2, "ldx": 127, "K": 127, **change}
        _expect(ctx, ctx._lib.esparse_mx_gemm(ctx._h, a["X"], a["xs"], a["M"], a["ldx"], a["act"], a["dtype"], a["w"], a["N"], a["K"], a["out"], a["Y"], a["ws"],
                                              a["nbytes"]), EWORKSPACE if a["ws"] else EINVAL, "workspace")


NORM = dict(x=P, ldx=64, r=None, ldr=0, w=P << 3, R=2, K=64, eps=1e-6, dtype=1, s=None, y=1 << 20, fmt=0, data=None, scales=None)


@pytest.mark.parametrize("change,code,word", [
    (dict(dtype=2), EUNSUPPORTED, "dtype"), (dict(R=-1), EINVAL, "rows"), (dict(K=0), EINVAL, "range"), (dict(eps=-1.0), EINVAL, "eps"), (dict(eps=math.nan), EINVAL, "eps"),
    (dict(x=None), EINVAL, "null"), (dict(w=None), EINVAL, "null"), (dict(y=None), EINVAL, "either"), (dict(data=P << 12, scales=P << 13), EINVAL, "either"),
    (dict(y=None, data=P << 12), EINVAL, "either"), (dict(y=None, data=P << 12, scales=P << 13, fmt=7), EUNSUPPORTED, "format"), (dict(ldx=63), EINVAL, "ldx"),
    (dict(r=P << 12, ldr=3), EINVAL, "ldr"), (dict(x=P + 1), EINVAL, "aligned"), (dict(y=P), EINVAL, "overlaps"), (dict(s=P + 2), EINVAL, "overlaps"),
    (dict(s=P, ldx=65), EINVAL, "overlaps"), (dict(s=1 << 20), EINVAL, "overlaps"), (dict(y=(P << 3) + 2), EINVAL, "overlaps"), (dict(s=(P << 3) - 2), EINVAL, "overlaps"), (dict(y=None, data=P << 12, scales=P << 12), EINVAL, "overlaps"), (dict(y=None, data=P + 128, scales=P << 13), EINVAL, "overlaps"),
    (dict(y=None, data=(P << 12) + 8, scales=P << 13), EINVAL, "16-byte")])
def test_norm_refuses(ctx, change, code, word):
    a = {**NORM, **change}
    _expect(ctx, ctx._lib.esparse_rms_norm(ctx._h, a["x"], a["ldx"], a["r"], a["ldr"], a["w"], a["R"], a["K"], a["eps"], a["dtype"], a["s"], a["y"], a["fmt"],
                                           a["data"], a["scales"]), code, word)


def test_rows_too_far_apart_are_refused(ctx):
    """Distances whose products with the rows pass 64 bits: a stretch of memory that seemed short before the check of overlaps."""
    for ld in ((1 << 62), (1 << 63) - 1, (1 << 38) + 1):
        _expect(ctx, ctx._lib.esparse_mx_quantize(ctx._h, P, 3, 8, ld, 0, 0, P << 4, P << 5), EINVAL, "out of range")
        for change in (dict(ldx=ld), dict(r=P << 12, ldr=ld)):
            a = {**NORM, "R": 3, **change}
            _expect(ctx, ctx._lib.esparse_rms_norm(ctx._h, a["x"], a["ldx"], a["r"], a["ldr"], a["w"], a["R"], a["K"], a["eps"], a["dtype"], a["s"], a["y"], a["fmt"],
                                                   a["data"], a["scales"]), EINVAL, "out of range")


LOGPROBS = dict(x=P, R=2, V=64, ld=64, dtype=1, tokens=P, top=0, lp=P, ent=P, ids=None, lps=None, ws=None, nbytes=0)


@pytest.mark.parametrize("change,code,word", [
    (dict(dtype=3), EUNSUPPORTED, "dtype"), (dict(V=(1 << 21) + 1, ld=1 << 22), EUNSUPPORTED, "V"), (dict(V=0), EINVAL, "range"), (dict(R=-1), EINVAL, "range"),
    (dict(top=-1), EINVAL, "top"), (dict(top=33), EINVAL, "top"), (dict(V=4, top=5), EINVAL, "top"), (dict(x=None), EINVAL, "null"), (dict(ld=63), EINVAL, "ld"),
    (dict(lp=None), EINVAL, "together"), (dict(tokens=None), EINVAL, "together"), (dict(top=2), EINVAL, "top_ids"), (dict(x=P + 1), EINVAL, "aligned"),
    (dict(tokens=P + 4), EINVAL, "aligned"), (dict(V=1 << 21, ld=1 << 21), EINVAL, "workspace"),
    (dict(V=1 << 21, ld=1 << 21, ws=P, nbytes=4), EWORKSPACE, "workspace"), (dict(V=1 << 21, ld=1 << 21, ws=P + 8, nbytes=1 << 30), EINVAL, "256-byte"),
    (dict(), EINVAL, "overlaps"), (dict(lp=P << 4, ent=P << 5, tokens=(P << 5) - 8), EINVAL, "overlaps"), (dict(lp=P << 4, ent=P + 128 + 124, tokens=P << 6), EINVAL, "overlaps"),
    (dict(lp=P << 4, ent=(P << 4) + 4, tokens=P << 6), EINVAL, "overlaps"), (dict(lp=P << 4, ent=P << 5, tokens=P << 6, top=2, ids=P << 7, lps=(P << 7) + 12), EINVAL, "overlaps"),
    (dict(lp=P << 4, ent=P << 5, tokens=P << 6, V=1 << 20, ld=1 << 20, x=1 << 30, ws=(1 << 30) + (1 << 20), nbytes=1 << 20), EINVAL, "overlaps")])
def test_logprobs_refuse(ctx, change, code, word):
    a = {**LOGPROBS, **change}
    _expect(ctx, ctx._lib.esparse_token_logprobs(ctx._h, a["x"], a["R"], a["V"], a["ld"], a["dtype"], a["tokens"], a["top"], a["lp"], a["ent"], a["ids"], a["lps"],
                                                 a["ws"], a["nbytes"]), code, word)


def test_nothing_to_do_needs_no_pointers(ctx):
    L, h = ctx._lib, ctx._h
    assert L.esparse_mx_quantize(h, None, 0, 8, 8, 0, 0, None, None) == 0
    assert L.esparse_mx_dequantize(h, None, None, 0, 8, 0, 0, None) == 0
    assert L.esparse_mx_gemm(h, None, None, 0, 8, 0, 0, None, 8, 8, 0, None, None, 0) == 0
    assert L.esparse_rms_norm(h, None, 8, None, 0, None, 0, 8, 1e-6, 0, None, None, 0, None, None) == 0
    assert L.esparse_token_logprobs(h, None, 0, 8, 8, 0, None, 0, None, None, None, None, None, 0) == 0
    for call in (lambda: L.esparse_mx_quantize(None, P, 1, 8, 8, 0, 0, P, P), lambda: L.esparse_mx_pack(None, P, P, 1, 8, P)):
        assert call() == EINVAL


# ---- refusals of the binding --------------------------------------------------------------------------
def test_binding_refuses(ctx):
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    mx = esp.MX(torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(1, 4, 4, dtype=torch.uint8), 64, esp.MX_FP4)
    w = esp.MXWeight(torch.zeros(esp.mx_packed_size(64, 64), dtype=torch.uint8), 64, 64)
    for call in (lambda: ctx.mx_quantize(x, esp.MX_FP4), lambda: ctx.mx_dequantize(mx), lambda: ctx.mx_pack(mx), lambda: ctx.mx_gemm(mx, w), lambda: ctx.mx_gemm(x, w),
                 lambda: ctx.rms_norm(x, x[0]), lambda: ctx.token_logprobs(x)):
        with pytest.raises(ValueError, match="on cpu, "):
            call()
    for call in (lambda: ctx.mx_quantize(x.double(), 0), lambda: ctx.mx_dequantize(mx, torch.float64), lambda: ctx.mx_gemm(x.float(), w),
                 lambda: ctx.rms_norm(x.float(), x[0]), lambda: ctx.token_logprobs(x.double())):
        with pytest.raises(TypeError):
            call()
