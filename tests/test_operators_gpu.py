"""The operators around a 4-bit linear layer on the GPU, against plain 64-bit implementations (oracle/operators_oracle.py).

Tolerances are derived, not fitted.  A rounding to 16 bits is off by at most half a step: 2^-8 (bf16), 2^-11 (f16) of the value.  A sum of n products
in fp32 is off by at most n 2^-23 times the sum of their magnitudes (one step of truncation for each addition).  With 8-bit activations the scaled matrix
instruction brings the products of eight consecutive channels to the largest of them, with exponent p, and cuts each to a multiple of 2^(p - 13): the seven
others lose less than 2^-13 of the largest each.
"""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2310_15929_amd as esp
from oracle import operators_oracle as orc

pytestmark = pytest.mark.gpu

TORCH = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}  # half a step of the smallest numbers
FMT = {"fp4": esp.MX_FP4, "fp8": esp.MX_FP8}


@pytest.fixture(scope="module")
def ctx():
    assert torch.cuda.is_available()
    return esp.Context(0)


def _rng(*key):
    return np.random.default_rng([int.from_bytes(str(k).encode(), "little") % (1 << 31) for k in key])


def _features(rng, R, K, dtype):
    x = rng.standard_normal((R, K)) * np.exp(rng.standard_normal(K))
    return torch.from_numpy(x).to(TORCH[dtype])


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _mx(x64, fmt):
    """(MX on the device, its values float64 [R, K]) from the oracle."""
    code, E = orc.mx_quantize(x64, fmt)
    return esp.MX(_dev(orc.mx_data(code, fmt)), _dev(orc.mx_scales(E)), x64.shape[1], fmt), orc.mx_values(code, E, fmt)[:, : x64.shape[1]]


def _assert_mx(got, x64, fmt, what=""):
    code, E = orc.mx_quantize(x64, fmt)
    assert np.array_equal(got.scales.cpu().numpy(), orc.mx_scales(E)), what
    assert np.array_equal(got.data.cpu().numpy(), orc.mx_data(code, fmt)), what


def _np(t):
    return t.double().cpu().numpy()


# ---- quantisation -----------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("R,K", [(1, 1), (1, 32), (3, 31), (2, 128), (17, 129), (16, 512), (33, 515), (5, 1000), (40, 4096)])
def test_quantize_codes_and_scales(ctx, R, K, dtype, fmt):
    x = _features(_rng(R, K, dtype, fmt), R, K, dtype)
    _assert_mx(ctx.mx_quantize(x.cuda(), FMT[fmt]), x.double().numpy(), FMT[fmt])


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_quantize_every_16_bit_value(ctx, dtype, fmt):
    """All finite values, each beside a largest value of every distance that matters: blocks of one value, its half, ... and the block's largest."""
    u = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(TORCH[dtype])
    u = u[torch.isfinite(u)]
    for shift in (0, 1, 3, 6, 10, 16):   # the block's largest value: the value times 2^shift, where that is one
        top = (u.double() * 2.0 ** shift).to(TORCH[dtype])
        top = torch.where(torch.isfinite(top), top, u)
        x = torch.zeros(u.numel(), 32, dtype=TORCH[dtype])
        x[:, 3], x[:, 30] = u, top
        x[:, 17] = (u.double() * -0.625).to(TORCH[dtype])
        x = x.reshape(-1, 128) if u.numel() % 4 == 0 else x
        _assert_mx(ctx.mx_quantize(x.cuda(), FMT[fmt]), x.double().numpy(), FMT[fmt], f"shift {shift}")


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_quantize_blocks_that_are_not_finite(ctx, dtype, fmt):
    x = _features(_rng("nan", dtype), 6, 200, dtype)
    x[0, 5], x[1, 40], x[2, 199], x[3, :] = math.nan, math.inf, -math.inf, 0.0
    q = ctx.mx_quantize(x.cuda(), FMT[fmt])
    _assert_mx(q, x.double().numpy(), FMT[fmt])
    v = _np(ctx.mx_dequantize(q, TORCH[dtype]))
    assert np.isnan(v[0, :32]).all() and np.isfinite(v[0, 32:]).all() and np.isnan(v[1, 32:64]).all() and np.isnan(v[2, 192:]).all()
    assert (v[3] == 0).all() and np.isfinite(v[4:]).all()


def test_quantize_f32_extremes(ctx):
    x = np.zeros((4, 128), np.float32)
    x[0, :4] = [1e-45, 3e-45, -1e-40, 1e-39]      # subnormal: the scale stays at 2^-127
    x[0, 32:35] = [3.4e38, -1e38, 1e30]
    x[1, 64:66] = [np.nextafter(np.float32(1), np.float32(0)), 2.0 ** -30]
    x[2, 0] = np.float32(2.0) ** -126
    x[3, 96] = -7.9
    for fmt in FMT.values():
        _assert_mx(ctx.mx_quantize(_dev(x), fmt), x.astype(np.float64), fmt)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("offset,ld", [(0, 300), (1, 301), (3, 517), (8, 264)])
def test_quantize_rows_apart_and_unaligned(ctx, dtype, offset, ld):
    K = 261
    base = _features(_rng("strided", ld), 1, 19 * ld + offset, dtype)[0].cuda()
    x = torch.as_strided(base, (19, K), (ld, 1), offset)
    _assert_mx(ctx.mx_quantize(x, esp.MX_FP8), x.double().cpu().numpy(), esp.MX_FP8)


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("R,K", [(1, 1), (3, 33), (18, 130), (5, 1003), (16, 2048)])
def test_dequantize(ctx, R, K, dtype, fmt):
    rng = _rng("read", R, K)
    q, want = _mx(rng.standard_normal((R, K)) * 10.0 ** rng.integers(-6, 4, (R, 1)), FMT[fmt])
    got = ctx.mx_dequantize(q, TORCH[dtype])
    assert torch.equal(got.cpu(), torch.from_numpy(want).to(TORCH[dtype]))


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_dequantize_every_code_and_scale(ctx, fmt):
    n = 16 if fmt == "fp4" else 256
    code = np.tile(np.arange(n, dtype=np.uint8), 256 * 256 // n).reshape(256, 256)
    E = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 8, 1)
    q = esp.MX(_dev(orc.mx_data(code, FMT[fmt])), _dev(orc.mx_scales(E)), 256, FMT[fmt])
    want = torch.from_numpy(orc.mx_values(code, E, FMT[fmt]))
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        got, w = ctx.mx_dequantize(q, dtype).cpu(), want.float().to(dtype)
        assert torch.equal(torch.isnan(got), torch.isnan(w)) and torch.equal(torch.nan_to_num(got, nan=1.0), torch.nan_to_num(w, nan=1.0))


# ---- product ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("N,K", [(1, 1), (16, 128), (17, 130), (64, 96), (100, 513), (200, 1024)])
def test_pack(ctx, N, K):
    x = _rng("pack", N, K).standard_normal((N, K))
    code, E = orc.mx_quantize(x, orc.FP4)
    got = ctx.mx_pack(_mx(x, orc.FP4)[0])
    assert (got.N, got.K) == (N, K) and np.array_equal(got.packed.cpu().numpy(), orc.mx_pack(code, E))


def _assert_product(got, x, w, dtype, act, what=""):
    """Each output is within its rounding and the error of a sum of K products in fp32, with 8-bit activations that of their products too."""
    want, size = x @ w.T, np.abs(x) @ np.abs(w).T
    before = (x.shape[1] + 16) * 2.0 ** -23 * size
    if act == "fp8":
        top = [np.abs(np.pad(v, ((0, 0), (0, -v.shape[1] % 8)))).reshape(v.shape[0], -1, 8).max(2) for v in (x, w)]
        before = before + 7 * 2.0 ** -13 * (top[0] @ top[1].T)
    bound = HALF[dtype] * np.abs(want) + before * (1 + HALF[dtype]) + TINY[dtype]
    err = np.abs(_np(got) - want)
    assert got.shape == want.shape and (err <= bound).all(), f"{what} {np.max(err / bound)} at {np.unravel_index(np.argmax(err / bound), err.shape)}"


def _product(ctx, M, N, K, act, dtype, out=None, seed=0):
    rng = _rng("product", M, N, K, act, dtype, seed)
    w, w64 = _mx(rng.standard_normal((N, K)) * K ** -0.5, orc.FP4)
    if act == "16":
        xt = _features(rng, M, K, dtype)
        X, x64 = xt.cuda(), xt.double().numpy()
    else:
        X, x64 = _mx(rng.standard_normal((M, K)) * np.exp(rng.standard_normal(K)), FMT[act])
    out = TORCH[out or dtype]
    _assert_product(ctx.mx_gemm(X, ctx.mx_pack(w), dtype=out), x64, w64, out, act, f"{M} x {N} x {K} {act}")


@pytest.mark.parametrize("act", ["16", "fp8", "fp4"])
@pytest.mark.parametrize("N,K", [(1, 1), (15, 32), (64, 128), (65, 100), (130, 257), (300, 1000), (512, 2048)])
@pytest.mark.parametrize("M", [1, 2, 7, 16, 17, 33, 64, 65, 130])
def test_product(ctx, M, N, K, act):
    _product(ctx, M, N, K, act, "bf16" if (M + N) % 2 else "f16")


@pytest.mark.parametrize("act", ["16", "fp8", "fp4"])
@pytest.mark.parametrize("M,N,K", [(256, 512, 640), (257, 1030, 384), (333, 1003, 620), (700, 2100, 1100), (1024, 1536, 512), (48, 5003, 3020), (3, 9000, 4096), (1, 22016, 1024)])
def test_product_larger(ctx, M, N, K, act):
    _product(ctx, M, N, K, act, "f16" if M % 2 else "bf16")


@pytest.mark.parametrize("act", ["16", "fp8", "fp4"])
@pytest.mark.parametrize("M,N,K", [(1, 4096, 4096), (1, 11008, 4096), (16, 22016, 8192), (32, 4096, 11008), (32, 22016, 8192), (64, 4096, 4096), (64, 11008, 4096), (64, 22016, 8192),
                                   (96, 5003, 3020), (128, 5120, 13824), (200, 9216, 9216), (333, 5003, 3020), (512, 13824, 5120), (768, 22016, 1024), (1024, 4096, 4096),
                                   (2048, 13824, 1280), (2048, 22016, 640), (1500, 1000, 900), (20, 11000, 640), (24, 5120, 640),
                                   (700, 18432, 640), (700, 18421, 1250), (1490, 13824, 4096), (512, 22016, 4096), (4, 5120, 384), (512, 11000, 512), (250, 22016, 384), (1, 1000, 4096), (2, 18432, 4000), (8, 22016, 640),
                                   (1, 4096, 11008)])
def test_product_of_layer_sizes(ctx, M, N, K, act):
    """Every kernel's own range of sizes; the 64-bit product is made on the device from the values read back (which other tests pin)."""
    gen = torch.Generator("cuda").manual_seed(M + N + K)
    wq = ctx.mx_quantize(torch.randn(N, K, device="cuda", generator=gen) * K ** -0.5, esp.MX_FP4)
    x = (torch.randn(M, K, device="cuda", generator=gen) * torch.exp(torch.randn(K, device="cuda", generator=gen))).bfloat16()
    X = x if act == "16" else ctx.mx_quantize(x, FMT[act])
    x64 = (x if act == "16" else ctx.mx_dequantize(X, torch.float32)).double()
    w64 = ctx.mx_dequantize(wq, torch.float32).double()
    got, want = ctx.mx_gemm(X, ctx.mx_pack(wq), dtype=torch.bfloat16).double(), x64 @ w64.t()
    before = (K + 16) * 2.0 ** -23 * (x64.abs() @ w64.abs().t())
    if act == "fp8":
        top = [torch.nn.functional.pad(v.abs(), (0, -K % 8)).reshape(v.shape[0], -1, 8).amax(2) for v in (x64, w64)]
        before += 7 * 2.0 ** -13 * (top[0] @ top[1].t())
    assert ((got - want).abs() <= 2.0 ** -8 * want.abs() + before * (1 + 2.0 ** -8)).all()


# a size for each kernel of the product, in the order of the tables in csrc/mx_matmul.hip, with odd numbers of features where that leaves the choice as it is
KERNEL_SIZES = {
    "fp8": [(1, 63, 128), (1, 4113, 128), (16, 20469, 133), (18, 61, 128), (24, 8267, 263), (33, 65, 128), (1, 8237, 128), (1, 63, 3604),
            (136, 67, 128), (587, 23365, 129), (1473, 13583, 129), (65, 8613, 1031), (534, 19621, 1033), (65, 4133, 392), (131, 63, 130)],
    "fp4": [(1, 64, 257), (1, 63, 129), (6, 16407, 129), (28, 61, 265), (17, 63, 128), (24, 8207, 129), (33, 63, 128), (1, 61, 128), (1, 64, 4612),
            (386, 23430, 129), (515, 22043, 1555), (66, 8253, 131), (518, 20397, 513), (2054, 193, 130), (130, 63, 133)],
    "16": [(1, 63, 129), (1, 4125, 129), (1, 63, 128), (6, 16415, 134), (18, 63, 129), (33, 65, 128),
           (274, 19750, 1430), (129, 22145, 672), (66, 16583, 128), (65, 17203, 515), (67, 1355, 2573), (17, 16653, 1161), (2059, 193, 129), (131, 65, 128), (65, 4197, 128)]}


@pytest.mark.parametrize("out", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("act,kernel", [(act, k) for act in KERNEL_SIZES for k in range(len(KERNEL_SIZES[act]))])
def test_product_of_each_kernel(ctx, act, kernel, dtype, out):
    """Every kernel with activations of both types (from both, if microscaled) and outputs of the three."""
    M, N, K = KERNEL_SIZES[act][kernel]
    gen = torch.Generator("cuda").manual_seed(M + N + K)
    wq = ctx.mx_quantize(torch.randn(N, K, device="cuda", generator=gen) * K ** -0.5, esp.MX_FP4)
    x = (torch.randn(M, K, device="cuda", generator=gen) * torch.exp(torch.randn(K, device="cuda", generator=gen))).to(TORCH[dtype])
    X = x if act == "16" else ctx.mx_quantize(x, FMT[act])
    x64 = (x if act == "16" else ctx.mx_dequantize(X, torch.float32)).double()
    w64 = ctx.mx_dequantize(wq, torch.float32).double()
    got, want = ctx.mx_gemm(X, ctx.mx_pack(wq), dtype=TORCH[out]), x64 @ w64.t()
    before = (K + 16) * 2.0 ** -23 * (x64.abs() @ w64.abs().t())
    if act == "fp8":
        top = [torch.nn.functional.pad(v.abs(), (0, -K % 8)).reshape(v.shape[0], -1, 8).amax(2) for v in (x64, w64)]
        before += 7 * 2.0 ** -13 * (top[0] @ top[1].t())
    half = HALF[TORCH[out]]
    assert got.dtype == TORCH[out] and ((got.double() - want).abs() <= half * want.abs() + before * (1 + half) + TINY[TORCH[out]]).all()


@pytest.mark.parametrize("act", ["16", "fp8", "fp4"])
@pytest.mark.parametrize("M", [1, 40, 300])
def test_product_of_the_most_channels(ctx, M, act):
    """K = 2^22, rows of 16 bits 2^23 bytes apart: offsets within a tile beyond 2^31.  200 channels of a token are no zeros, so that the bound of the sums stays small."""
    gen = torch.Generator("cuda").manual_seed(M)
    N, K, n = 40, 1 << 22, 200
    wq = ctx.mx_quantize(torch.randn(N, K, device="cuda", generator=gen).bfloat16(), esp.MX_FP4)
    at = (torch.arange(n, device="cuda") * 20971 + torch.arange(M, device="cuda")[:, None] * 977) % K
    at[:, 0], at[:, 1] = 0, K - 1
    assert (at.sort(1).values.diff(dim=1) > 0).all()
    x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda").scatter_(1, at, torch.randn(M, n, device="cuda", generator=gen).bfloat16())
    X = x if act == "16" else ctx.mx_quantize(x, FMT[act])
    got = ctx.mx_gemm(X, ctx.mx_pack(wq), dtype=torch.float32).double()
    values = (x if act == "16" else ctx.mx_dequantize(X, torch.bfloat16)).gather(1, at).double()
    w = ctx.mx_dequantize(wq, torch.float32)
    want, size = torch.empty(M, N, dtype=torch.float64, device="cuda"), torch.empty(M, N, dtype=torch.float64, device="cuda")
    for m in range(M):
        p = w[:, at[m]].double() * values[m]
        want[m], size[m] = p.sum(1), p.abs().sum(1)
    # sums of n products (zeros add nothing); 8 bits: a product alone among its eight channels is not cut, one beside a larger one by less than 2^-13 of that
    before = (n + 16) * 2.0 ** -23 * size + (7 * 2.0 ** -13 * size if act == "fp8" else 0)
    assert ((got - want).abs() <= before * (1 + HALF[torch.float32]) + HALF[torch.float32] * want.abs()).all()


@pytest.mark.parametrize("act", ["16", "fp8", "fp4"])
@pytest.mark.parametrize("M,N", [(5, 70), (40, 96), (140, 131), (300, 640), (200, 640), (513, 1000), (1030, 2100), (2050, 4100)])
def test_product_in_32_bits(ctx, M, N, act):
    _product(ctx, M, N, 520, act, "f16", out="f32")


@pytest.mark.parametrize("dtype,out", [("f16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("M,N", [(200, 64), (64, 130), (20, 130), (200, 4090), (33, 11000)])
@pytest.mark.parametrize("K", [1, 128, 200, 384, 520, 640, 900])
def test_product_with_k_in_halves(ctx, M, N, K, dtype, out):
    """Two groups of waves share the 128-channel steps of K: none for the second, as many for both, one less; K not a multiple of 128."""
    _product(ctx, M, N, K, "16", dtype, out=out)


@pytest.mark.parametrize("act", ["16", "fp8", "fp4"])
@pytest.mark.parametrize("M,N,K", [(20, 130, 2800), (20, 64, 3200), (33, 500, 4600), (100, 11000, 3100), (333, 4090, 3100)])
def test_product_with_k_cut_unevenly(ctx, M, N, K, act):
    """A last piece of K with a single step of 128 channels, among others."""
    _product(ctx, M, N, K, act, "bf16")


@pytest.mark.parametrize("M", [1, 20, 150])
def test_product_of_each_type_pair(ctx, M):
    """16-bit activations of one type, outputs of the other."""
    _product(ctx, M, 192, 256, "16", "f16", out="bf16")
    _product(ctx, M, 192, 256, "16", "bf16", out="f16")


@pytest.mark.parametrize("M", [1, 16, 40, 200])
@pytest.mark.parametrize("offset,ld", [(0, 264), (1, 257), (8, 300), (4, 1000)])
def test_product_rows_apart_and_unaligned(ctx, M, offset, ld):
    rng, K, N = _rng("rows", M, ld), 256, 80
    base = _features(rng, 1, M * ld + offset, "bf16")[0].cuda()
    x = torch.as_strided(base, (M, K), (ld, 1), offset)
    w, w64 = _mx(rng.standard_normal((N, K)), orc.FP4)
    _assert_product(ctx.mx_gemm(x, ctx.mx_pack(w)), _np(x), w64, torch.bfloat16, "16")


@pytest.mark.parametrize("act", ["16", "fp8", "fp4"])
@pytest.mark.parametrize("M", [1, 30, 150])
def test_product_of_bad_blocks_stays_in_their_rows(ctx, M, act):
    """A NaN scale reaches the outputs of its row and of its token only; a padded tail holds none."""
    rng, N, K = _rng("bad", M), 70, 290
    x, w = rng.standard_normal((M, K)), rng.standard_normal((N, K))
    w[3, 200], x[M - 1, 289] = math.nan, math.nan
    wq, w64 = _mx(w, orc.FP4)
    if act == "16":
        xt = torch.from_numpy(x).bfloat16()
        X, x64 = xt.cuda(), xt.double().numpy()
    else:
        X, x64 = _mx(x, FMT[act])
    got = _np(ctx.mx_gemm(X, ctx.mx_pack(wq), dtype=torch.float32))
    bad = np.zeros((M, N), bool)
    bad[:, 3] = bad[M - 1] = True
    assert np.array_equal(np.isnan(got), bad)
    _assert_product(torch.from_numpy(np.where(bad, 0, got)[:, 4:]).float(), np.nan_to_num(x64) * (np.arange(M) < M - 1)[:, None], w64[4:], torch.float32, act)


def test_product_with_wide_scales(ctx):
    """Scales from 2^-60 to 2^60 in weights and activations: no block's products disturb another's."""
    rng, M, N, K = _rng("wide"), 20, 48, 384
    x = rng.standard_normal((M, K)) * np.ldexp(1.0, rng.integers(-30, 30, (M, K // 32))).repeat(32, 1)
    w = rng.standard_normal((N, K)) * np.ldexp(1.0, rng.integers(-30, 30, (N, K // 32))).repeat(32, 1)
    wq, w64 = _mx(w, orc.FP4)
    for act in ("fp8", "fp4"):
        X, x64 = _mx(x, FMT[act])
        _assert_product(ctx.mx_gemm(X, ctx.mx_pack(wq), dtype=torch.float32), x64, w64, torch.float32, act, act)
    xt = torch.from_numpy(x).bfloat16()
    _assert_product(ctx.mx_gemm(xt.cuda(), ctx.mx_pack(wq), dtype=torch.float32), xt.double().numpy(), w64, torch.float32, "16", "16")


@pytest.mark.parametrize("act", ["f16", "bf16", "fp8", "fp4"])
@pytest.mark.parametrize("M", [1, 16, 50, 200, 600])
def test_product_of_every_code_and_scale(ctx, M, act):
    """Weights of one number a row, all codes with all scales, times 1: in 16 bits the weight as a conversion to that type gives it (f16: exact for scales of 2^-23 to 2^13,
    rounded to even below, infinite beyond 65504), with microscaled activations as fp32 holds it."""
    K = 256
    E = np.repeat(np.arange(255, dtype=np.uint8), 16)[:, None].repeat(K // 32, 1)
    code = np.zeros((len(E), K), np.uint8)
    code[np.arange(len(E)), np.arange(len(E)) * 37 % K] = np.tile(np.arange(16, dtype=np.uint8), 255)
    w = orc.mx_values(code, E, orc.FP4).sum(1)
    packed = ctx.mx_pack(esp.MX(_dev(orc.mx_data(code, orc.FP4)), _dev(orc.mx_scales(E)), K, esp.MX_FP4))
    ones = torch.ones(M, K, dtype=TORCH[act] if act in TORCH else torch.float32, device="cuda")
    y = ctx.mx_gemm(ones if act in TORCH else ctx.mx_quantize(ones, FMT[act]), packed, dtype=torch.float32).cpu()
    want = torch.from_numpy(w).to(TORCH.get(act, torch.float32)).float()
    if act == "f16":
        s = np.repeat(np.arange(255) - 127, 16)
        inside = torch.from_numpy((s >= -23) & (s <= 13))
        assert torch.equal(want[inside].double(), torch.from_numpy(w)[inside]) and torch.isinf(want[(np.abs(w) > 65504).nonzero()[0]]).all()
    assert torch.equal(y, want.expand(M, -1))


@pytest.mark.parametrize("M", [1, 16, 200])
def test_product_of_weights_beyond_f16(ctx, M):
    """A weight beyond 65504 is infinite for f16 activations: the output of its row is infinite, NaN opposite a zero; bf16 activations take it as it is; other rows stay as they are."""
    rng, K, N = _rng("beyond f16", M), 256, 80
    w = rng.standard_normal((N, K))
    w[7, 100] = 98304.0     # 6 x 2^14
    x = rng.standard_normal((M, K))
    x[0, 100] = 0.0
    x[1:, 100] = 0.5 + np.abs(x[1:, 100])
    wq, w64 = _mx(w, orc.FP4)
    xt = torch.from_numpy(x)
    y = ctx.mx_gemm(xt.half().cuda(), ctx.mx_pack(wq), dtype=torch.float32)
    assert torch.isnan(y[0, 7]) and (y[1:, 7] == math.inf).all()
    keep = np.arange(N) != 7
    _assert_product(y[:, torch.from_numpy(keep).cuda()], xt.half().double().numpy(), w64[keep], torch.float32, "16")
    _assert_product(ctx.mx_gemm(xt.bfloat16().cuda(), ctx.mx_pack(wq), dtype=torch.float32), xt.bfloat16().double().numpy(), w64, torch.float32, "16")


@pytest.mark.parametrize("M,N,K", [(1, 300, 4096), (16, 512, 2048), (40, 1000, 1100), (333, 1003, 620), (700, 2100, 1100)])
def test_product_of_8_bit_activations_with_full_sums(ctx, M, N, K):
    """MX 8-bit values are exact in bf16: read back and multiplied as 16-bit activations they give the sums in fp32 that the scaled instruction cuts (its products of eight
    consecutive channels at 2^-13 of the largest)."""
    rng = _rng("full sums", M, N)
    w, w64 = _mx(rng.standard_normal((N, K)) * K ** -0.5, orc.FP4)
    x = rng.standard_normal((M, K)) * np.exp(2 * rng.standard_normal(K))
    X, x64 = _mx(x, orc.FP8)
    packed = ctx.mx_pack(w)
    back = ctx.mx_dequantize(X, torch.bfloat16)
    assert np.array_equal(_np(back), x64)
    _assert_product(ctx.mx_gemm(X, packed, dtype=torch.float32), x64, w64, torch.float32, "fp8")
    _assert_product(ctx.mx_gemm(back, packed, dtype=torch.float32), x64, w64, torch.float32, "16")


def test_product_leaves_other_memory_alone(ctx):
    """Guards around the output and behind the workspace keep their pattern, whatever part of a tile is used."""
    for M, N, K, act in [(1, 5, 40, "16"), (19, 33, 130, "fp8"), (70, 129, 300, "16"), (150, 257, 256, "fp4"), (260, 300, 1000, "fp8"), (300, 1001, 333, "16")]:
        rng = _rng("guard", M, N)
        w, w64 = _mx(rng.standard_normal((N, K)), orc.FP4)
        X, x64 = (_features(rng, M, K, "f16").cuda(), None) if act == "16" else _mx(rng.standard_normal((M, K)), FMT[act])
        buf = torch.full((M * N + 512,), 7.25, dtype=torch.float16, device="cuda")
        y = buf[256:256 + M * N].view(M, N)
        ctx.mx_gemm(X, ctx.mx_pack(w), out=y, dtype=torch.float16)
        assert (buf[:256] == 7.25).all() and (buf[256 + M * N:] == 7.25).all()
        _assert_product(y, _np(X) if act == "16" else x64, w64, torch.float16, act)


@pytest.mark.parametrize("M", [1, 9, 40, 200, 300])
def test_product_reads_nothing_behind_a_row(ctx, M):
    """16-bit rows with NaN and infinities between them and behind the last: K a multiple of 8, of 128, of neither."""
    for K, ld in ((200, 208), (256, 264), (136, 136), (1000, 1024), (77, 80)):
        rng = _rng("behind", M, K)
        base = torch.full((M * ld + 256,), math.nan, dtype=torch.bfloat16, device="cuda")
        base[1::3] = math.inf
        x = torch.as_strided(base, (M, K), (ld, 1))
        x.copy_(_features(rng, M, K, "bf16"))
        w, w64 = _mx(rng.standard_normal((90, K)), orc.FP4)
        _assert_product(ctx.mx_gemm(x, ctx.mx_pack(w)), _np(x), w64, torch.bfloat16, "16", f"{M} {K} {ld}")


def test_product_is_the_same_every_time(ctx):
    for M, N, K in [(3, 4096, 4096), (40, 512, 4096), (333, 1003, 1000)]:
        x = _features(_rng("again", M), M, K, "bf16").cuda()
        w = ctx.mx_pack(_mx(_rng("again w", N).standard_normal((N, K)), orc.FP4)[0])
        first = ctx.mx_gemm(x, w)
        assert all(torch.equal(first, ctx.mx_gemm(x, w)) for _ in range(3))


# ---- norm -------------------------------------------------------------------------------------------
def _norm_bound(y, K, half, tiny):
    # sum of K squares (relative K 2^-23), its root halves that; root, division, two products: 2^-24 each and the sum's division
    return np.abs(y) * (half + K * 2.0 ** -24 + 6 * 2.0 ** -24) + tiny


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("R,K", [(1, 1), (1, 8), (5, 31), (3, 512), (70, 513), (2, 2048), (3, 4097), (300, 4096), (2, 8192), (3, 13824), (2, 16385), (2, 33000)])
def test_norm(ctx, R, K, residual, dtype):
    rng = _rng("norm", R, K)
    x, r = _features(rng, R, K, dtype), _features(rng, R, K, dtype)
    w = torch.from_numpy(rng.standard_normal(K)).to(TORCH[dtype])
    y, h = ctx.rms_norm(x.cuda(), w.cuda(), 1e-5, residual=r.cuda() if residual else None)
    h64 = (x.double() + r.double()).to(TORCH[dtype]).double() if residual else x.double()
    assert torch.equal(h.double().cpu(), h64)
    want = orc.rms_norm(h64.numpy(), w.double().numpy(), 1e-5)
    assert (np.abs(_np(y) - want) <= _norm_bound(want, K, HALF[TORCH[dtype]], TINY[TORCH[dtype]])).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("R,K", [(300, 4096), (70, 8192), (900, 1000), (20, 33000)])
def test_norm_to_mx_rounds_once(ctx, R, K, fmt, dtype):
    """The codes of the exact norm, all of them: sums in 64 bits, and results that are not exact kept off the middles between two codes
    (eps is a power of two: it is the same number in 32 bits and in 64)."""
    rng = _rng("norm once", R, K)
    x, r = _features(rng, R, K, dtype), _features(rng, R, K, dtype)
    w = torch.from_numpy(rng.standard_normal(K)).to(TORCH[dtype])
    q, _ = ctx.rms_norm(x.cuda(), w.cuda(), 2.0 ** -17, residual=r.cuda(), fmt=FMT[fmt])
    h64 = (x.double() + r.double()).to(TORCH[dtype]).double().numpy()
    _assert_mx(q, orc.rms_norm(h64, w.double().numpy(), 2.0 ** -17), FMT[fmt])


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("K", [64, 512, 4096, 33024])
def test_norm_right_on_the_middle_of_two_codes(ctx, K, fmt):
    """Rows whose norm is rational and no power of two: y is exact there, and the weights put it on the middles between codes, beside them, and on powers of two."""
    rng = _rng("norm middle", K)
    mid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 1.0, 2.0, 4.0, 6.0, 1.0078125, 0.99609375, 2.515625, 2.484375])
    if fmt == "fp8":
        mid = np.concatenate([mid, np.array([(2 * m + 1) / 16 * 2.0 ** e for m in range(8, 16) for e in (-2, 0, 3)])])
    w = torch.from_numpy(mid[rng.integers(0, len(mid), K)] * np.where(rng.random(K) < 0.5, -1.0, 1.0)).bfloat16()
    sign = np.where(rng.random((40, K)) < 0.5, -1.0, 1.0)
    size = np.array([1.0, 3, 5, 7, 11, 13, 49, 77, 101, 127])[np.arange(40) % 10] * np.array([1.0, 0.125, 2.0 ** 12, 2.0 ** -13])[np.arange(40) // 10]
    x = torch.from_numpy(sign * size[:, None]).bfloat16()
    want = orc.rms_norm(x.double().numpy(), w.double().numpy(), 0.0)
    assert np.array_equal(np.abs(want), np.broadcast_to(np.abs(w.double().numpy()), want.shape))   # exact in 64 bits
    _assert_mx(ctx.rms_norm(x.cuda(), w.cuda(), 0.0, fmt=FMT[fmt])[0], want, FMT[fmt])
    # several magnitudes: of 64 channels 15 are 3, one is 21: a mean square of 9 (15 + 49) / 64 = 9
    pattern = np.zeros(64)
    pattern[3::4] = 3.0
    pattern[7] = 21.0
    x = torch.from_numpy(np.tile(pattern, K // 64)[None] * sign[:3]).bfloat16()
    want = orc.rms_norm(x.double().numpy(), w.double().numpy(), 0.0)
    assert np.array_equal(want, x.double().numpy() / 3 * w.double().numpy())
    _assert_mx(ctx.rms_norm(x.cuda(), w.cuda(), 0.0, fmt=FMT[fmt])[0], want, FMT[fmt])


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("K", [64, 520, 4096, 33000])
def test_norm_beside_the_middle_of_two_codes(ctx, K, fmt):
    """Rows of ones with an eps that takes y as little as 2^-51 below weights that are on middles and powers of two; of 3 with an eps for the same."""
    rng = _rng("norm beside", K)
    mid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 1.0, 2.0, 4.0, 6.0] + ([(2 * m + 1) / 16 for m in range(8, 16)] if fmt == "fp8" else []))
    w = torch.from_numpy(mid[rng.integers(0, len(mid), K)] * np.where(rng.random(K) < 0.5, -1.0, 1.0)).bfloat16()
    for size in (1.0, 3.0):
        x = torch.from_numpy(size * np.where(rng.random((5, K)) < 0.5, -1.0, 1.0)).bfloat16()
        for bits in (30, 40, 44, 47, 50):
            want = orc.rms_norm(x.double().numpy(), w.double().numpy(), size * size * 2.0 ** -bits)
            assert (np.abs(want) < np.abs(w.double().numpy())).all()
            _assert_mx(ctx.rms_norm(x.cuda(), w.cuda(), size * size * 2.0 ** -bits, fmt=FMT[fmt])[0], want, FMT[fmt], f"{size} {bits}")


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("K", [100, 225, 900, 4500, 14400, 40000])
def test_norm_right_on_the_middle_where_the_mean_is_no_number_of_64_bits(ctx, K, fmt):
    """36 or 64 of 100 channels of one magnitude, the others 0: a root mean square of 0.6 or 0.8 of it, and weights that put weight / 0.6 or weight / 0.8 on middles."""
    rng = _rng("norm fraction", K)
    for part, (num, den) in ((0.36, (5, 3)), (0.64, (5, 4))):
        on = np.arange(K) < round(K * part)
        sign = np.where(rng.random((9, K)) < 0.5, -1.0, 1.0) * rng.permuted(np.broadcast_to(on, (9, K)), axis=1)
        base = np.array([1.0, 1.25, 1.625, 0.5, 2.0, 4.0, 1.9375]) * (den / 4 if den == 4 else 0.75)
        w = base[rng.integers(0, len(base), K)] * np.where(rng.random(K) < 0.5, -1.0, 1.0)
        x = sign * np.array([1.0, 3, 5, 7, 11, 2.0 ** -9, 96, 13, 0.625])[:, None]
        want = np.abs(sign) * sign * (w * num / den)[None]    # in numbers of a few bits: exact
        xt, wt = torch.from_numpy(x).bfloat16(), torch.from_numpy(w).bfloat16()
        assert np.array_equal(xt.double().numpy(), x) and np.array_equal(wt.double().numpy(), w) and (want * 1024 % 1 == 0).all()
        assert np.allclose(want, orc.rms_norm(x, w, 0.0), rtol=1e-14, atol=0)
        _assert_mx(ctx.rms_norm(xt.cuda(), wt.cuda(), 0.0, fmt=FMT[fmt])[0], want, FMT[fmt])


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_norm_takes_eps_in_64_bits(ctx, fmt):
    """Rows whose mean square is of the size of eps, which is no 32-bit number."""
    rng, R, K = _rng("norm eps"), 200, 4096
    x = (_features(rng, R, K, "bf16").double() * 2.0 ** -9).bfloat16()
    w = torch.from_numpy(rng.standard_normal(K)).bfloat16()
    q, _ = ctx.rms_norm(x.cuda(), w.cuda(), 1.1e-5, fmt=FMT[fmt])
    _assert_mx(q, orc.rms_norm(x.double().numpy(), w.double().numpy(), 1.1e-5), FMT[fmt])


@pytest.mark.parametrize("R,K", [(5, 100), (5, 4096), (5, 33000)])
def test_norm_of_rows_that_are_no_numbers(ctx, R, K):
    rng = _rng("norm nan", K)
    x, w = _features(rng, R, K, "bf16"), torch.ones(K, dtype=torch.bfloat16)
    x[1, K // 2], x[2, 3], x[3] = float("nan"), float("-inf"), 0.0
    y, _ = ctx.rms_norm(x.cuda(), w.cuda(), 1e-5)
    y = y.cpu()
    assert torch.isnan(y[1]).all() and torch.isnan(y[2, 3]) and torch.isnan(y[2]).sum() == 1 and (y[2][~torch.isnan(y[2])] == 0).all() and (y[3] == 0).all()
    assert torch.isfinite(y[[0, 4]]).all() and torch.isnan(ctx.rms_norm(x.cuda(), w.cuda(), 0.0)[0][3]).all()
    q, _ = ctx.rms_norm(x.cuda(), w.cuda(), 1e-5, fmt=esp.MX_FP8)
    v = ctx.mx_dequantize(q, torch.float32).cpu()
    assert torch.isnan(v[1]).all() and torch.isnan(v[2, :32]).all() and (v[2, 32:] == 0).all() and (v[3] == 0).all() and torch.isfinite(v[[0, 4]]).all()


@pytest.mark.parametrize("fmt", [None, "fp4", "fp8"])
def test_norm_of_rows_whose_squares_pass_32_bits(ctx, fmt):
    rng, K = _rng("norm far"), 520
    x = (_features(rng, 6, K, "f16").double() * 2.0 ** torch.tensor([[0.0], [64], [100], [-70], [-100], [30]], dtype=torch.float64)).bfloat16()
    w = torch.from_numpy(rng.standard_normal(K)).bfloat16()
    want = orc.rms_norm(x.double().numpy(), w.double().numpy(), 2.0 ** -17)
    y, _ = ctx.rms_norm(x.cuda(), w.cuda(), 2.0 ** -17, fmt=fmt and FMT[fmt])
    if fmt:
        _assert_mx(y, want, FMT[fmt])
    else:
        assert (np.abs(_np(y) - want) <= _norm_bound(want, 0, HALF[torch.bfloat16], TINY[torch.bfloat16])).all()


@pytest.mark.parametrize("fmt", [None, "fp4", "fp8"])
@pytest.mark.parametrize("K", [64, 520, 4100, 8200, 33000])
def test_norm_of_rows_whose_inverse_passes_32_bits(ctx, K, fmt):
    """Rows from the smallest bf16 numbers to the largest, eps 0 or of their size: 1 / rms up to 2^133, down to 2^-127, and h weight beyond fp32 in either direction."""
    rng = _rng("norm inverse", K)
    for row_exp, w_exp, eps in ((-133, 0, 0.0), (-129, 0, 0.0), (-127, 3, 2.0 ** -260), (-100, -30, 0.0), (-61, -90, 0.0), (-59, 0, 0.0), (59, 0, 0.0), (61, 60, 0.0), (110, 100, 0.0), (125, 0, 0.0), (125, 2, 2.0 ** 300)):
        x = torch.from_numpy(rng.integers(1, 8, (3, K)) * np.where(rng.random((3, K)) < 0.5, -1.0, 1.0) * 2.0 ** (row_exp - (0 if row_exp < 0 else 2))).bfloat16()
        w = torch.from_numpy((1 + rng.random(K)) * 2.0 ** w_exp).bfloat16()
        assert (x != 0).all() and torch.isfinite(x).all()
        want = orc.rms_norm(x.double().numpy(), w.double().numpy(), eps)
        y, _ = ctx.rms_norm(x.cuda(), w.cuda(), eps, fmt=fmt and FMT[fmt])
        if fmt:
            _assert_mx(y, want, FMT[fmt], f"{row_exp} {w_exp}")
        else:  # one rounding of a value that is right to 2^-23
            bound = np.abs(want) * (HALF[torch.bfloat16] + 2.0 ** -23) + TINY[torch.bfloat16]
            assert (np.abs(_np(y) - want) <= bound).all(), (row_exp, w_exp)
    # f16 rows with an eps that takes y below every f16 number, but not below every scale
    x = torch.from_numpy(rng.standard_normal((2, K))).half()
    w = torch.from_numpy(1 + rng.random(K)).half()
    y, _ = ctx.rms_norm(x.cuda(), w.cuda(), 2.0 ** 140, fmt=fmt and FMT[fmt])
    if fmt:
        _assert_mx(y, orc.rms_norm(x.double().numpy(), w.double().numpy(), 2.0 ** 140), FMT[fmt])
    else:
        assert (y == 0).all()
    # one value that is no zero among many: 1 / rms above it by the root of K
    x = torch.zeros(2, K, dtype=torch.bfloat16)
    x[0, K // 2], x[1, 1] = 2.0 ** -133, -2.0 ** 127
    w = torch.full((K,), 1.5, dtype=torch.bfloat16)
    want = orc.rms_norm(x.double().numpy(), w.double().numpy(), 0.0)
    y, _ = ctx.rms_norm(x.cuda(), w.cuda(), 0.0, fmt=fmt and FMT[fmt])
    if fmt:
        _assert_mx(y, want, FMT[fmt])
    else:
        assert (np.abs(_np(y) - want) <= np.abs(want) * (HALF[torch.bfloat16] + 2.0 ** -23)).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("R,K", [(1, 1), (5, 33), (3, 512), (70, 515), (20, 4096), (3, 4097), (2, 13824), (2, 33000)])
def test_norm_to_mx(ctx, R, K, fmt, dtype):
    """The codes are those of the exact norm, but where the sum's rounding moves a value across the middle of two of them or a block's largest across a power of two."""
    rng = _rng("norm mx", R, K)
    x, r = _features(rng, R, K, dtype), _features(rng, R, K, dtype)
    w = torch.from_numpy(rng.standard_normal(K)).to(TORCH[dtype])
    q, h = ctx.rms_norm(x.cuda(), w.cuda(), 1e-5, residual=r.cuda(), fmt=FMT[fmt])
    h64 = (x.double() + r.double()).to(TORCH[dtype]).double().numpy()
    want = orc.rms_norm(h64, w.double().numpy(), 1e-5)
    off = K * 2.0 ** -24 + 6 * 2.0 ** -24
    got = _np(ctx.mx_dequantize(q, torch.float32))
    lo, hi = (np.stack([orc.mx_values(*orc.mx_quantize(want * (1 + d), FMT[fmt]), FMT[fmt])[:, :K] for d in (-off, 0.0, off)]) for _ in range(2))
    lo, hi = lo.min(0), hi.max(0)
    assert ((got >= lo) & (got <= hi)).all()
    # the channels behind the last are zeros
    kp = q.data.shape[1] * (2 if fmt == "fp4" else 1)
    tail = ctx.mx_dequantize(esp.MX(q.data, q.scales, kp, FMT[fmt]), torch.float32)[:, K:]
    assert (tail == 0).all()


def test_norm_in_place_and_rows_apart(ctx):
    rng, R, K = _rng("place"), 21, 700
    x, r = _features(rng, R, K, "bf16").cuda(), _features(rng, R, K, "bf16").cuda()
    w = torch.from_numpy(rng.standard_normal(K)).bfloat16().cuda()
    y, h = ctx.rms_norm(x, w, residual=r)
    for where in ("x", "residual"):
        a, b = x.clone(), r.clone()
        y2, h2 = ctx.rms_norm(a, w, residual=b, sum_out=a if where == "x" else b)
        assert torch.equal(h2, h) and torch.equal(y2, y) and torch.equal(b if where == "x" else a, r if where == "x" else x)
    wide = torch.zeros(R, 1501, dtype=torch.bfloat16, device="cuda")
    wide[:, 3:703], wide[:, 801:1501] = x, r
    y2, h2 = ctx.rms_norm(wide[:, 3:703], w, residual=wide[:, 801:1501])
    assert torch.equal(h2, h) and torch.equal(y2, y)
    assert ctx.rms_norm(x, w)[1] is x
    with pytest.raises(esp.EsparseError, match="overlaps"):
        ctx.rms_norm(x[:-1], w, residual=r[:-1], sum_out=x[1:])


@pytest.mark.parametrize("fmt", [None, "fp8"])
@pytest.mark.parametrize("K", [64, 700, 33000])
def test_norm_without_a_residual_keeps_its_input(ctx, K, fmt):
    """sum_out without a residual receives x; x itself may be it."""
    rng = _rng("copy", K)
    x, w = _features(rng, 5, K, "f16").cuda(), torch.from_numpy(rng.standard_normal(K)).half().cuda()
    wide = torch.zeros(5, K + 3, dtype=torch.float16, device="cuda")
    wide[:, 1:K + 1] = x
    y, h = ctx.rms_norm(x, w, fmt=fmt and FMT[fmt])
    kept, same = torch.full_like(x, 7.0), x.clone()
    for y2, h2 in (ctx.rms_norm(wide[:, 1:K + 1], w, fmt=fmt and FMT[fmt], sum_out=kept), ctx.rms_norm(same, w, fmt=fmt and FMT[fmt], sum_out=same)):
        assert torch.equal(h2, x) and h is x
        assert torch.equal(y2.data, y.data) and torch.equal(y2.scales, y.scales) if fmt else torch.equal(y2, y)
    assert h2 is same and torch.equal(kept, x)


def test_norm_of_extreme_rows(ctx):
    w = torch.ones(256, dtype=torch.bfloat16, device="cuda")
    x = torch.ones(5, 256, dtype=torch.bfloat16, device="cuda")
    x[0], x[1, 7], x[2, 7], x[3] = 0, math.nan, math.inf, 2.0 ** -100
    y = ctx.rms_norm(x, w, 1e-6)[0].float().cpu()
    assert (y[0] == 0).all() and torch.isnan(y[1]).all() and torch.isnan(y[2, 7]) and (y[2, :7] == 0).all() and (y[4] == 1).all()
    assert torch.allclose(y[3], torch.full((256,), 2.0 ** -100 * 1000.0), rtol=0.01, atol=0)
    q = ctx.rms_norm(x, w, 1e-6, fmt=esp.MX_FP8)[0]
    v = ctx.mx_dequantize(q, torch.float32).cpu()
    assert (v[0] == 0).all() and torch.isnan(v[1]).all() and torch.isnan(v[2, :32]).all() and (v[2, 32:] == 0).all()
    # a row of zeros without eps: 0 times infinity, in the row's channels and not in the padding
    q = ctx.rms_norm(torch.zeros(2, 40, dtype=torch.bfloat16, device="cuda"), w[:40].contiguous(), 0.0, fmt=esp.MX_FP8)[0]
    assert torch.isnan(ctx.mx_dequantize(q, torch.float32)).all() and (q.scales.cpu()[0, :, 2:] == 0).all()


# ---- log probabilities ------------------------------------------------------------------------------
def _assert_logprobs(ctx, x, tokens, top, what=""):
    x64 = x.double().cpu().numpy()
    lp, ent, ids, tops = orc.token_logprobs(x64, tokens, top)
    r = ctx.token_logprobs(x, torch.tensor(tokens, dtype=torch.int64, device="cuda"), top=top)
    V = x.shape[1]
    # ln s: the terms' errors (exp 2^-22, its argument |d| 2^-23 with p |d| at most 0.37) and the sum's, 2 ln2(V) 2^-24 relative as a tree over runs of 128
    s_err = 2.0 ** -21 + (128 + 2 * math.log2(V + 1)) * 2.0 ** -24
    def bound(v):
        return s_err + 4 * 2.0 ** -24 * (np.abs(v) + 32)
    def check(got, want, tol):
        assert np.array_equal(np.isnan(got), np.isnan(want)), what
        fine = np.isfinite(want)
        assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), what
        assert (np.abs(got - want)[fine] <= tol[fine]).all(), (what, np.max((np.abs(got - want) / tol)[fine]))
    check(_np(r.logprob), lp, bound(np.nan_to_num(lp, posinf=0, neginf=0)))
    # t / s: each term's p d is off by p |d| times the same, the sum of p |d| / s is at most ln V
    check(_np(r.entropy), ent, bound(np.nan_to_num(ent)) + s_err * (2 + 2 * math.log(V + 1)))
    if top:
        assert np.array_equal(r.top_ids.cpu().numpy(), ids), what
        check(_np(r.top_logprobs), tops, bound(np.nan_to_num(tops, posinf=0, neginf=0)))
    else:
        assert r.top_ids is None and r.top_logprobs is None


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("R,V,top", [(1, 1, 1), (3, 2, 2), (2, 31, 20), (5, 100, 32), (4, 1000, 5), (1, 5003, 0), (7, 16384, 20), (3, 32000, 1), (2, 50021, 32),
                                     (8, 131072, 20), (1, 131073, 3), (2, 300001, 20), (40, 8191, 7), (300, 4099, 4)])
def test_logprobs(ctx, R, V, top, dtype):
    rng = _rng("lp", R, V, top)
    x = torch.from_numpy(rng.standard_normal((R, V)) * 3).to(TORCH[dtype]).cuda()
    _assert_logprobs(ctx, x, [int(t) for t in rng.integers(0, V, R)], top)


@pytest.mark.parametrize("V", [40, 5000, 70000, 140000])
def test_logprobs_of_masked_rows(ctx, V):
    """Minus infinity in places, everywhere, everywhere but one; infinities and NaN; equal values; padding and foreign tokens."""
    rng = _rng("mask", V)
    for dtype in ("f16", "bf16", "f32"):
        x = torch.from_numpy(rng.standard_normal((12, V)) * 2).to(TORCH[dtype])
        x[0, rng.random(V) < 0.7] = -math.inf
        x[1] = -math.inf
        x[2] = -math.inf
        x[2, V // 2] = -5.0
        x[3, V - 1] = math.nan
        x[4, 3] = math.inf
        x[5] = 1.5
        x[6] = torch.where(torch.arange(V) % 3 == 0, 2.0, -1.0).to(TORCH[dtype])
        x[7] = 0.0
        x[7, 5] = -0.0
        x[8] = torch.finfo(TORCH[dtype]).min
        x[9, :] = math.nan
        x[10, 1] = -math.nan
        x[11, V - 3:] = 60.0
        tokens = [0, 1, V // 2, 0, 1, 2, -1, -100, 7, 3, 0, V]
        _assert_logprobs(ctx, x.cuda(), tokens, min(20, V), f"{V} {dtype}")
        _assert_logprobs(ctx, x.cuda(), [t - 1 if 0 < t < V else t for t in tokens], 1, f"{V} {dtype}")


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("R,V", [(1, 7), (3, 40), (2, 5000), (1100, 3000), (3, 70000), (2, 140000)])
def test_logprobs_of_rows_of_negative_nan(ctx, R, V, dtype):
    """A NaN of either sign makes the row NaN and all its ids -1, however few other values there are: outputs that held something else before."""
    bits = {"f16": -0x200, "bf16": -0x40, "f32": -0x400000}[dtype]   # the quiet NaN with the sign set
    for finite in (0, 1, 3, V - 1):
        x = torch.full((R, V), bits, dtype=torch.int32 if dtype == "f32" else torch.int16).view(TORCH[dtype]).clone()
        x[0, V - finite:] = torch.arange(finite).to(TORCH[dtype]) / 8
        assert torch.isnan(x[:, 0]).all() and torch.signbit(x[:, 0]).all()
        for top in {1, min(5, V), min(32, V)}:
            code = {"f16": esp.F16, "bf16": esp.BF16, "f32": esp.F32}[dtype]
            nbytes = esp.token_logprobs_workspace(R, V, code, top)
            ws = torch.zeros(nbytes + 1, dtype=torch.uint8, device="cuda")
            dev, tok = x.cuda(), torch.full((R,), V - 1, device="cuda")
            ids, tops, lp, ent = (torch.full(shape, 777, dtype=t, device="cuda")
                                  for shape, t in (((R, top), torch.int32), ((R, top), torch.float32), ((R,), torch.float32), ((R,), torch.float32)))
            ctx._sync_stream()
            assert ctx._lib.esparse_token_logprobs(ctx._h, dev.data_ptr(), R, V, V, code, tok.data_ptr(), top, lp.data_ptr(), ent.data_ptr(), ids.data_ptr(), tops.data_ptr(),
                                                   ws.data_ptr(), nbytes) == 0
            assert (ids == -1).all() and torch.isnan(tops).all() and torch.isnan(lp).all() and torch.isnan(ent).all(), (finite, top)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("R,V", [(13, 300), (13, 5000), (13, 16376), (13, 70001), (1050, 9001), (13, 140000)])
def test_logprobs_of_rows_with_many_equal_values(ctx, R, V, dtype):
    """Rows in which a mask leaves none to 40 values (minus infinity, the type's lowest number, a large negative one), rows of two and three values, ties between the alternatives,
    and a few threads' values above all others: more of them than a workgroup lists."""
    rng = _rng("equal", R, V)
    low = {"f16": -65504.0, "bf16": float(torch.finfo(torch.bfloat16).min), "f32": float(torch.finfo(torch.float32).min)}[dtype]
    x = np.full((13, V), -math.inf)
    for r, (fill, count) in enumerate(((-math.inf, 1), (-math.inf, 5), (-math.inf, 19), (-math.inf, 40), (low, 0), (low, 5), (low, 33), (-10000.0, 3), (-10000.0, 21))):
        x[r] = fill
        x[r, rng.permutation(V)[:count]] = rng.standard_normal(count) * 3
    x[9] = np.where(rng.random(V) < 0.3, 1.0, 0.5)                                          # thousands tie for the first places
    x[10] = np.where(rng.random(V) < 12 / V, 2.0, np.where(rng.random(V) < 0.4, -1.0, -3.0))  # a dozen first, then ties
    x[11] = np.where(np.arange(V) // (4 if dtype == "f32" else 8) % 256 < 31, rng.standard_normal(V), -5.0)   # 31 threads of 256 hold all but one value
    x[12] = np.where(np.arange(V) < V - 7, -2.5, 1.0)                                       # the last ones first, then from the start
    x = torch.from_numpy(x).to(TORCH[dtype])
    x = torch.cat((x, x[torch.arange(R - 13) % 13])).cuda()
    tokens = torch.arange(R, device="cuda") * 7919 % V
    for top in (1, 5, 20, 32):
        _assert_logprobs(ctx, x[:13], [int(t) for t in tokens[:13]], top, f"{dtype} {top}")
        if R > 13:   # one workgroup a row
            few, many = ctx.token_logprobs(x[:13], tokens[:13], top=top), ctx.token_logprobs(x, tokens, top=top)
            assert all(torch.equal(many.top_ids[i:i + 13], few.top_ids) for i in range(0, R - 13, 13))


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("R", [1, 40, 1100])
def test_logprobs_of_the_largest_vocabulary(ctx, R, dtype):
    """V = 2^21: rows cut into 32 pieces, into 25, and not at all."""
    V = 1 << 21
    x = torch.randn(min(R, 3), V, device="cuda", generator=torch.Generator("cuda").manual_seed(R)).mul_(3).to(TORCH[dtype])
    x[0, -1], x[0, 0], x[-1, V // 2:] = 20.0, 20.0, -math.inf
    tokens = [V - 1] + [V // 2 - 1] * (R - 1)
    if R > 3:
        first = _np(x)
        r = ctx.token_logprobs(x[torch.arange(R, device="cuda") % 3], torch.tensor(tokens, device="cuda"), top=32)
        lp, ent, ids, tops = orc.token_logprobs(first, tokens[:3], 32)
        s_err = 2.0 ** -21 + (128 + 2 * 21) * 2.0 ** -24
        for row in (0, 1, 2, R - 3, R - 2, R - 1):
            assert np.array_equal(r.top_ids[row].cpu().numpy(), ids[row % 3])
            assert (np.abs(_np(r.top_logprobs[row]) - tops[row % 3]) <= s_err + 4 * 2.0 ** -24 * (np.abs(tops[row % 3]) + 32)).all()
            assert abs(float(r.entropy[row]) - ent[row % 3]) <= s_err * (3 + 2 * math.log(V)) + 4 * 2.0 ** -24 * (ent[row % 3] + 32)
    else:
        _assert_logprobs(ctx, x, tokens, 32)


def test_logprobs_far_from_zero(ctx):
    """A common offset of the logits takes no precision beyond that of the logits themselves."""
    rng = _rng("far")
    x = torch.from_numpy(rng.standard_normal((6, 9000)) * 3 + np.array([0, 1e3, -1e3, 3e4, -3e4, 1e5])[:, None]).float()
    _assert_logprobs(ctx, x.cuda(), [5] * 6, 8)


def test_logprobs_rows_apart_and_unaligned(ctx):
    rng, V = _rng("lp rows"), 3001
    for dtype in ("f16", "bf16", "f32"):
        base = torch.from_numpy(rng.standard_normal(9 * 3333 + 5)).to(TORCH[dtype]).cuda()
        for offset in (0, 1, 3):
            _assert_logprobs(ctx, torch.as_strided(base, (9, V), (3333, 1), offset), list(range(9)), 6, f"{dtype} {offset}")


def test_logprobs_without_tokens(ctx):
    x = torch.randn(3, 500, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    r = ctx.token_logprobs(x, top=2)
    assert r.logprob is None and torch.equal(r.top_ids.long(), torch.topk(x, 2).indices)


def test_logprobs_do_not_depend_on_other_rows(ctx):
    gen = torch.Generator("cuda").manual_seed(2)
    for R, V in ((700, 3000), (5, 40000)):
        x = torch.randn(R, V, device="cuda", generator=gen)
        t = torch.arange(R, device="cuda")
        first = ctx.token_logprobs(x, t, top=5)
        x[1::2] = torch.randn(R // 2, V, device="cuda", generator=gen) * 50
        x[1, 3] = math.nan
        second = ctx.token_logprobs(x, t, top=5)
        for a, b in zip((first.logprob, first.entropy, first.top_ids, first.top_logprobs), (second.logprob, second.entropy, second.top_ids, second.top_logprobs)):
            assert torch.equal(a[::2], b[::2])


@pytest.mark.parametrize("R,V,dtype", [(8, 131072, "bf16"), (1, 8192, "f16"), (1, 32000, "bf16"), (3, 70000, "f32"), (2000, 3000, "f16")])
def test_logprobs_order_of_the_sums(ctx, R, V, dtype):
    """How many alternatives are asked for does not change a row's sums; whether any are may, in the last bits."""
    x = torch.from_numpy(_rng("order", R, V).standard_normal((R, V)) * 3).to(TORCH[dtype]).cuda()
    tokens = torch.arange(R, device="cuda")
    results = [ctx.token_logprobs(x, tokens, top=top) for top in (0, 1, 5, 32)]
    for r in results[2:]:
        assert torch.equal(r.logprob, results[1].logprob) and torch.equal(r.entropy, results[1].entropy)
        assert torch.equal(r.top_ids[:, :1], results[1].top_ids) and torch.equal(r.top_logprobs[:, :1], results[1].top_logprobs)
    _assert_logprobs(ctx, x[:8], list(range(min(R, 8))), 0)
    # both are within the bound of test_logprobs for a row's sum of the exact value
    s_err = 2.0 ** -21 + (128 + 2 * math.log2(V + 1)) * 2.0 ** -24
    assert ((results[0].logprob - results[1].logprob).abs() <= 2 * (s_err + 4 * 2.0 ** -24 * (results[0].logprob.abs() + 32))).all()


# ---- beyond 32 bits -----------------------------------------------------------------------------------
def test_offsets_beyond_32_bits(ctx):
    """The last rows of matrices with more than 2^32 bytes and values are those of a call on these rows alone."""
    gen = torch.Generator("cuda").manual_seed(9)
    R, K, last = 70000, 65536, 5
    x = torch.empty(R, K, dtype=torch.bfloat16, device="cuda")
    x.normal_(generator=gen)
    tail = x[-last:].clone()
    for fmt in FMT.values():
        q, part = ctx.mx_quantize(x, fmt), ctx.mx_quantize(tail, fmt)
        assert torch.equal(q.data[-last:], part.data) and torch.equal(q.scales[:, -last:], part.scales)
        assert torch.equal(ctx.mx_dequantize(q, torch.bfloat16)[-last:], ctx.mx_dequantize(part, torch.bfloat16))
    w = torch.ones(K, dtype=torch.bfloat16, device="cuda")
    y, h = ctx.rms_norm(x, w, residual=x)
    y2, h2 = ctx.rms_norm(tail, w, residual=tail)
    assert torch.equal(y[-last:], y2) and torch.equal(h[-last:], h2)
    del y, h, q
    big, small = ctx.token_logprobs(x, torch.arange(R, device="cuda"), top=3), ctx.token_logprobs(tail, torch.arange(R - last, R, device="cuda") % K, top=3)
    assert torch.equal(big.top_ids[-last:], small.top_ids) and torch.allclose(big.entropy[-last:], small.entropy, rtol=1e-5)
    # outputs of a product beyond 2^32: 70000 tokens x 65600 features of 128 channels
    a, b = ctx.mx_quantize(x[:, :128], esp.MX_FP8), ctx.mx_quantize(x[:65600, 128:256], esp.MX_FP4)
    packed = ctx.mx_pack(b)
    out = ctx.mx_gemm(a, packed)
    alone = ctx.mx_gemm(ctx.mx_quantize(tail[:, :128], esp.MX_FP8), packed)
    assert torch.equal(out[-last:], alone)
    out = ctx.mx_gemm(x[:, :128], packed)
    assert torch.allclose(out[-last:].float(), ctx.mx_gemm(tail[:, :128].contiguous(), packed).float(), rtol=2.0 ** -7, atol=1e-3)


# ---- empty inputs -------------------------------------------------------------------------------------
def test_no_rows(ctx):
    x = torch.zeros(0, 64, dtype=torch.bfloat16, device="cuda")
    w = ctx.mx_pack(ctx.mx_quantize(torch.ones(8, 64, dtype=torch.bfloat16, device="cuda"), esp.MX_FP4))
    q = ctx.mx_quantize(x, esp.MX_FP8)
    assert ctx.mx_dequantize(q).shape == (0, 64) and ctx.mx_gemm(q, w).shape == (0, 8) and ctx.mx_gemm(x, w).shape == (0, 8)
    assert ctx.rms_norm(x, torch.ones(64, dtype=torch.bfloat16, device="cuda"), residual=x)[0].shape == (0, 64)
    r = ctx.token_logprobs(x, torch.zeros(0, dtype=torch.int64, device="cuda"), top=3)
    assert r.logprob.shape == (0,) and r.top_ids.shape == (0, 3)


# ---- refusals of the binding --------------------------------------------------------------------------
def test_binding_refuses(ctx):
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    mx = ctx.mx_quantize(x, esp.MX_FP4)
    w = ctx.mx_pack(mx)
    tok = torch.zeros(4, dtype=torch.int64, device="cuda")
    for call in (lambda: ctx.mx_quantize(x.t(), 0), lambda: ctx.mx_quantize(x[0], 0), lambda: ctx.mx_quantize(x[:1].expand(4, 64), 0), lambda: ctx.mx_quantize(x, 2),
                 lambda: ctx.mx_dequantize(esp.MX(mx.data, mx.scales, 200, 0)), lambda: ctx.mx_dequantize(esp.MX(mx.data, mx.scales, 64, 1)),
                 lambda: ctx.mx_dequantize(esp.MX(mx.data.char(), mx.scales, 64, 0)), lambda: ctx.mx_dequantize(esp.MX(mx.data, mx.scales, 64, 5)),
                 lambda: ctx.mx_dequantize(esp.MX(mx.data, mx.scales.transpose(0, 1), 64, 0)), lambda: ctx.mx_pack(ctx.mx_quantize(x, esp.MX_FP8)),
                 lambda: ctx.mx_gemm(x[:, :32], w), lambda: ctx.mx_gemm(x, esp.MXWeight(w.packed[:-1], 4, 64)), lambda: ctx.mx_gemm(x, esp.MXWeight(w.packed, 4, 200)),
                 lambda: ctx.mx_gemm(x, w, out=x), lambda: ctx.mx_gemm(x, w, out=x[:, :4]), lambda: ctx.mx_gemm(x, w, out=torch.empty(4, 4, device="cuda"), dtype=torch.float16),
                 lambda: ctx.rms_norm(x, x[0, :32]), lambda: ctx.rms_norm(x, x[0].float()), lambda: ctx.rms_norm(x, x[0], residual=x[:2]), lambda: ctx.rms_norm(x, x[0], fmt=3),
                 lambda: ctx.rms_norm(x, x[0], sum_out=torch.zeros(4, 128, dtype=torch.bfloat16, device="cuda")[:, :64]),
                 lambda: ctx.token_logprobs(x, tok.int()), lambda: ctx.token_logprobs(x, tok[:3]), lambda: ctx.rms_norm(x, x[0].cpu()), lambda: ctx.token_logprobs(x, tok.cpu())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: ctx.token_logprobs(x, tok, top=33), lambda: ctx.token_logprobs(x, tok, top=-1), lambda: ctx.token_logprobs(x[:, :4], tok, top=5),
                 lambda: ctx.rms_norm(x, x[0], math.nan), lambda: ctx.rms_norm(x, x[0], -1.0)):
        with pytest.raises(esp.EsparseError):
            call()


# ---- together, as they are used -----------------------------------------------------------------------
def _run_together(ctx, x, residual, norm_w, layer, head, tokens):
    """Residual and norm into 8 bits, a 4-bit layer, norm, the vocabulary's product in 32 bits, log probabilities."""
    q, h = ctx.rms_norm(x, norm_w, 1e-5, residual=residual, fmt=esp.MX_FP8)
    z = ctx.mx_gemm(q, layer, dtype=x.dtype)
    y, h = ctx.rms_norm(z, norm_w, 1e-5, residual=h)
    logits = ctx.mx_gemm(y, head, dtype=torch.float32)
    r = ctx.token_logprobs(logits, tokens, top=5)
    return r.logprob, r.entropy, r.top_ids, r.top_logprobs, logits, h


def _together_inputs(ctx, M, K=512, V=3000):
    rng = _rng("together", M)
    x, r = _features(rng, M, K, "bf16").cuda(), _features(rng, M, K, "bf16").cuda()
    nw = torch.from_numpy(1 + 0.2 * rng.standard_normal(K)).bfloat16().cuda()
    wl, wh = (torch.from_numpy(rng.standard_normal((n, K)) * K ** -0.5).bfloat16().cuda() for n in (K, V))
    layer, head = (ctx.mx_pack(ctx.mx_quantize(w, esp.MX_FP4)) for w in (wl, wh))
    return x, r, nw, layer, head, torch.from_numpy(rng.integers(0, V, M)).cuda(), wl, wh


@pytest.mark.parametrize("M", [1, 20, 300])
def test_together(ctx, M):
    """Each step against 64 bits from the device's own input of that step."""
    x, r, nw, layer, head, tokens, wl, wh = _together_inputs(ctx, M)
    lp, ent, ids, tops, logits, h = _run_together(ctx, x, r, nw, layer, head, tokens)
    q, h1 = ctx.rms_norm(x, nw, 1e-5, residual=r, fmt=esp.MX_FP8)
    w64 = [orc.mx_values(*orc.mx_quantize(w.double().cpu().numpy(), orc.FP4), orc.FP4) for w in (wl, wh)]
    z = ctx.mx_gemm(q, layer, dtype=torch.bfloat16)
    _assert_product(z, _np(ctx.mx_dequantize(q, torch.float32)), w64[0], torch.bfloat16, "fp8")
    y, h2 = ctx.rms_norm(z, nw, 1e-5, residual=h1)
    assert torch.equal(h, h2)
    _assert_product(logits, _np(y), w64[1], torch.float32, "16")
    _assert_logprobs(ctx, logits, [int(t) for t in tokens], 5)
    again = ctx.token_logprobs(logits, tokens, top=5)
    assert torch.equal(again.logprob, lp) and torch.equal(again.entropy, ent) and torch.equal(again.top_ids, ids) and torch.equal(again.top_logprobs, tops)


@pytest.mark.parametrize("M", [1, 40, 260])
def test_captured_and_replayed(ctx, M):
    """Two graphs of the same calls, replayed in turn with eager work between, give what eager calls give on the inputs of the moment."""
    x, r, nw, layer, head, tokens, *_ = _together_inputs(ctx, M)
    _run_together(ctx, x, r, nw, layer, head, tokens)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        ins = [x.clone(), r.clone(), tokens.clone()]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = _run_together(ctx, ins[0], ins[1], nw, layer, head, ins[2])
        graphs.append((g, ins, outs))
    gen = torch.Generator("cuda").manual_seed(3)
    for turn in range(4):
        for g, ins, outs in graphs:
            ins[0].copy_(torch.randn(x.shape, device="cuda", generator=gen))
            ins[2].copy_(torch.randint(0, 3000, tokens.shape, device="cuda", generator=gen))
            g.replay()
            want = _run_together(ctx, ins[0], ins[1], nw, layer, head, ins[2])
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, want)), turn


def test_on_other_streams(ctx):
    """Calls on a stream that is not the default one, and two contexts on two streams at once."""
    x, r, nw, layer, head, tokens, *_ = _together_inputs(ctx, 33)
    want = _run_together(ctx, x, r, nw, layer, head, tokens)
    other = esp.Context(0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    results = []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            results.append(_run_together((ctx, other)[i % 2], x, r, nw, layer, head, tokens))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for res in results for a, b in zip(res, want))
