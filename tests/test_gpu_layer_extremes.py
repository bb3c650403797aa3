"""Epilogues, their gradient and what else stands around the products, far out: at the lowest and the largest numbers, infinities and NaN.

Bounds that do not grow with |p|, u = 2^-24.
  SiLU's slope, q (1 + c k), e = e^-c, q = 1 / (1 + e), k = e q, c = p but no less than -88.  e is off by (1.23 |c| + 4) u of itself (the exponent's
  rounding and its constant's, 2 ulp of the power), and of q by at most the share e / (1 + e) of that, 3 u more from the sum and the reciprocal (1 ulp).
  c >= 0: |c| e <= 0.37, so q is within 7.5 u; c k <= 0.28 and within 4.6 u; the slope, at most 1.28 times 9.5 u and 4.6 u: 17 u.
  c < 0: q <= e^-|c| and within (1.23 |c| + 7) u, e^-|c| (1 + |c|) (1.23 |c| + 10) <= 10.1; k's share, q |c| times what e leaves in e / (1 + e) and
  3 u, below 3 u: 14 u.  24 u for both, and below -88 less than 89 e^-88 < 6e-37.
  GELU_TANH's slope, (1 + t) / 2 + A (1 - t^2), t = tanh(a), r = sqrt(2 / pi) c, a = r + 0.044715 r c^2, A = 3 a / 2 - r, c = p within 16 of
  zero.  1 - t^2 is off by 2 |t| times t's error and by one rounding.  Up to a = 0.6 t is within 8 u of itself and A <= 0.33: 5.2 u and a
  third of that.  From there on t is off by half a step, u / 2, and by (1 - t) (2 a + 8) u, and a's four roundings add (1 - t^2) a 4 u, which
  together stay below 6 u and below u / 2 + 0.1 u from c = 3 on, while A is 0.5, 2.7, 9.7 at c = 1, 3, 5.2.  Beyond 5.2 t is 1.  That is 11 u
  at c = 5.2, where 1 - t^2 is nothing, and 4 u at c = 1.  A is within 15 u of itself, and A (1 - t^2) <= 0.3: 5 u.  The first summand is
  within 4 u, the last sum, of at most 1.13, rounds once more: 24 u.
The sum over N columns in a tree whose longest path is one thread's share: (N / 32 + 32) u of the sum of magnitudes.
"""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import layer_oracle as lo
from test_gpu_layers import B, BF16, F32, KERNELS, U, close, dev, num  # noqa: F401  (B: the fixture)
from workloads import generators as gen

pytestmark = pytest.mark.gpu

LOWEST = {F32: float(np.finfo(np.float32).min), BF16: -3.3895313892515355e38}
FAR = [0.0, -0.0, 1e-38, -1e-38, 1.0, -1.0, 79.5, -79.5, 80.5, -80.5, 87.0, -87.0, 88.0, -88.0, 88.5, -88.5, 100.0, -100.0, 1e4, -1e4, 1e19, -1e19, 1e20,
       -1e20, 1e28, -1e28, 1e30, -1e30, 1e35, -1e35]


def slope_case(B, act, dtype, N, slope_bound, limits):
    """Rows whose P holds one far value in some places among ordinary ones; limits: the slope at -infinity and infinity (NaN
    where the formula is 0 times infinity), and at NaN where that is a number."""
    values = FAR + [LOWEST[dtype], -LOWEST[dtype]]
    M = len(values) + 3
    g = np.random.default_rng(N)
    P, DY = dev(2 * g.normal(size=(M, N)), dtype), dev(g.normal(size=(M, N)), dtype)
    at = sorted({0, 5 % N, N // 2, N - 1})
    for r, v in enumerate(values + [-np.inf, np.inf, np.nan]):
        P[r, at] = v
    p, dy = num(P), num(DY)
    finite = np.arange(M) < len(values)
    want = dy.copy()
    want[finite] *= lo.act_grad(act, p[finite])
    rest = np.setdiff1d(np.arange(N), at)
    for r, v in zip((M - 3, M - 2, M - 1), (*limits, np.nan)):
        want[r, rest] *= lo.act_grad(act, p[r, rest])
        want[r, at] *= v
    bound = slope_bound * np.abs(dy)
    for out in ("new", "dY", "pre", None):
        dY, pre = DY.clone(), P.clone()
        dP = {"new": torch.empty_like(DY), "dY": dY, "pre": pre, None: None}[out]
        db = torch.empty(M, device="cuda")
        B.grim_epilogue_grad(dY, dP, lo.ACTS.index(act), pre, db)
        whole = ~np.isnan(want)
        rows = whole.all(1)
        if dP is not None:
            got = num(dP)
            assert np.array_equal(np.isnan(got), ~whole)
            close(got[whole], want[whole], bound[whole], dtype, "dP")
        s = num(db)
        assert np.array_equal(np.isnan(s), ~rows)
        close(s[rows], want[rows].sum(1), bound[rows].sum(1) + (N / 32 + 32) * U * np.abs(want[rows]).sum(1), F32, "dbias")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N", [1, 7, 333, 4100])
def test_slope_of_silu_far_out(B, dtype, N):  # noqa: F811
    slope_case(B, "silu", dtype, N, 24 * U, (0.0, np.nan))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N", [1, 7, 333, 4100])
def test_slope_of_gelu_tanh_far_out(B, dtype, N):  # noqa: F811
    slope_case(B, "gelu_tanh", dtype, N, 24 * U, (0.0, 1.0))


@pytest.mark.parametrize("bf16", [False, True])
def test_products_refuse_operands_between_elements(B, bf16):  # noqa: F811
    """Refused on the host: nothing is launched, nothing written."""
    M, K, N, dt, esz = 32, 16, 24, BF16 if bf16 else F32, 2 if bf16 else 4
    h = B.grim_bcr_pack(np.ones((M, K), np.float32), np.ones((M, K), np.uint8), 4, 16, int(bf16), 0)
    buf = {k: torch.full((M * N + 8,), 3.0, device="cuda", dtype=dt) for k in "XYRP"}
    bias = torch.zeros(M + 2, device="cuda")
    torch.cuda.synchronize()
    before = B.grim_launch_count()
    for off in range(1, esz):
        for which in ("X", "Y", "R", "P", "bias"):
            mat = {k: B.grim_mat_t(t.data_ptr() + (off if k == which else 0), K if k == "X" else M, N, N, int(bf16)) for k, t in buf.items()}
            x, y, r, p = (C.byref(mat[k]) for k in "XYRP")
            e = B.grim_epilogue_t(bias.data_ptr() + (off if which == "bias" else 0), B.GRIM_ACT_SILU, C.pointer(mat["R"]), C.pointer(mat["P"]))
            tune = B.grim_tune_t()
            got = [B.lib.grim_bcr_linear(h, x, C.byref(e), y, None), B.lib.grim_bcr_linear_ex(h, x, C.byref(e), y, C.byref(tune), None)]
            if which in "XY":
                got += [B.lib.grim_bcr_spmm(h, x, y, None), B.lib.grim_bcr_spmm_ex(h, x, y, C.byref(tune), None)]
            assert got == [B.GRIM_ERR_INVALID_ARG] * len(got), (which, off, got)
    assert B.grim_launch_count() == before
    torch.cuda.synchronize()
    assert all((t == 3.0).all() for t in buf.values())
    assert B.grim_bcr_status(h) == B.GRIM_OK
    B.grim_bcr_destroy(h)


@pytest.mark.parametrize("act", lo.ACTS)
@pytest.mark.parametrize("kernel", KERNELS, ids=[k[0] for k in KERNELS])
def test_activations_far_out_in_every_kernel(B, kernel, act):  # noqa: F811
    """X = 0, so that p is the bias: y is within 8 u of itself and 32 u, whatever p; sigmoids stop at 1.8e-35."""
    _, size, choice = kernel
    s = dict(bf16=False, **size) if "bf16" not in size else size
    M, K, N, bf16 = s["M"], s["K"], s["N"], s["bf16"]
    W = gen.dense_weight(M, K, seed=21)
    h = B.grim_bcr_pack(W, gen.bcr_mask(M, K, s["bh"], s["bw"], compression=s["rate"], dist="uniform", seed=22, stream=3), s["bh"], s["bw"], int(bf16), 0)
    if bf16:
        B.grim_bcr_reserve(h, N)
    X = torch.zeros(K, N, device="cuda", dtype=BF16 if bf16 else F32)
    for yt in ((BF16, F32) if bf16 else (F32,)):
        values = FAR + [LOWEST[yt], -LOWEST[yt], np.inf, -np.inf, np.nan]
        b = np.resize(np.asarray(values, np.float32), M)
        R = torch.randn(M, N, device="cuda").to(yt)
        Y, P = torch.empty(M, N, device="cuda", dtype=yt), torch.empty(M, N, device="cuda", dtype=yt)
        B.grim_bcr_linear(h, X, Y, dev(b), lo.ACTS.index(act), R, P, **choice)
        with np.errstate(invalid="ignore", over="ignore"):
            y = lo.act(act, b.astype(np.float64))[:, None]
        if act == "relu":
            y = np.where(np.isnan(b[:, None]), np.nan, y)
        want = y + num(R)
        got = num(Y)
        sure = np.isfinite(want)
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
        close(got[sure], want[sure], (32 * U + 8 * U * np.abs(want) + 1e-34)[sure], yt, "Y")
        assert torch.equal(torch.nan_to_num(P), torch.nan_to_num(dev(b)[:, None].expand(M, N).to(yt))) and torch.equal(torch.isnan(P), torch.isnan(dev(b))[:, None].expand(M, N))
    assert B.grim_bcr_status(h) == B.GRIM_OK
    B.grim_bcr_destroy(h)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "sigmoid", "tanh"])
def test_other_slopes_far_out(B, act, dtype):  # noqa: F811
    """GELU's slope, Phi(p) + p e / sqrt(2 pi), e = e^(-p^2 / 2): e's exponent rounds by up to 1.2 p^2 u and its power by 4 u, and
    p e <= 0.61, p^3 e <= 1.16, so the second summand is within 0.4 (1.2 * 1.16 + 6 * 0.61) u < 2.1 u; Phi is within 4.2 u; one fma: 10 u.
    sigmoid's, q k <= 1/4, each within (1.23 |p| + 8) u of itself, |p| q k <= 0.23: 6 u; tanh's, 1 - t^2: 16 u and a rounding.  24 u for all."""
    for N in (1, 7, 333, 4100):
        slope_case(B, act, dtype, N, 24 * U, {"gelu": (np.nan, np.nan), "none": (1.0, 1.0, 1.0), "relu": (0.0, 1.0, 0.0)}.get(act, (0.0, 0.0)))
