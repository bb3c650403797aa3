"""The calls around the products as programs make them: into parts of larger allocations, captured into graphs, on other streams, and the
gradient to X with transposed handles.  Bounds: those of test_gpu_layers.py."""
import numpy as np
import pytest
import torch

from oracle import bcr_oracle as orc
from oracle import layer_oracle as lo
from test_gpu_layers import B, BF16, F32, KERNELS, U, close, dev, num, place  # noqa: F401  (B: the fixture)
from workloads import generators as gen

pytestmark = pytest.mark.gpu

MARK = 55.0


def framed(rows, cols, dtype, ld=None, shift=0):
    """A matrix inside an allocation full of MARK, and a check that nothing beside it was written."""
    ld = cols if ld is None else ld
    m, whole = place(rows, cols, dtype, ld, shift, MARK)

    def untouched():
        beside = torch.ones_like(whole, dtype=torch.bool)
        beside[shift:shift + rows * ld].view(rows, ld)[:, :cols] = False
        return bool((whole[beside] == MARK).all())
    return m, untouched


# ---------------------------------------------------------------------------------------- beside the outputs

@pytest.mark.parametrize("ld,shift", [(0, 0), (3, 1), (8, 8)])
@pytest.mark.parametrize("kernel", KERNELS, ids=[k[0] for k in KERNELS])
def test_linear_writes_its_outputs_alone(B, kernel, ld, shift):  # noqa: F811
    """P has a stride and stores of its own in every kernel."""
    _, s, choice = kernel
    M, K, N, bf16 = s["M"], s["K"], s["N"], s.get("bf16", False)
    W, X, b = gen.dense_weight(M, K, seed=31), gen.normal_f32((K, N), 1.0, 33, 1), gen.normal_f32((M,), 0.5, 33, 2)
    mask = gen.bcr_mask(M, K, s["bh"], s["bw"], compression=s["rate"], dist="uniform", seed=32, stream=3)
    X = gen.bf16_representable(X) if bf16 else X
    Wm = orc.masked_weight(W, mask, int(bf16))
    p = Wm @ X.astype(np.float64) + b[:, None]
    scale = np.linalg.norm(Wm, axis=1)[:, None] * np.linalg.norm(X.astype(np.float64), axis=0)[None, :] + np.abs(b)[:, None]
    h = B.grim_bcr_pack(W, mask, s["bh"], s["bw"], int(bf16), 0)
    if bf16:
        B.grim_bcr_reserve(h, N)
    for yt in ((BF16, F32) if bf16 else (F32,)):
        Y, beside_y = framed(M, N, yt, N + ld, shift)
        P, beside_p = framed(M, N, yt, N + 2 * ld, shift)
        B.grim_bcr_linear(h, dev(X, BF16 if bf16 else F32), Y, dev(b), B.GRIM_ACT_SILU, None, P, **choice)
        close(P, p, 1e-5 * scale, yt, "pre")
        close(Y, lo.act("silu", p), 1.13 * 1e-5 * scale + 32 * U * (1 + np.abs(p)), yt, "Y")
        assert beside_y() and beside_p()
    assert B.grim_bcr_status(h) == B.GRIM_OK
    B.grim_bcr_destroy(h)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("H,N,starts", [(10, 777, [2, 300, 301, 770]), (3, 5003, None), (300, 1200, [0, 0, 700, 1200, 1200]), (2, 20011, [5, 9000, 20000])])
@pytest.mark.parametrize("ld,shift", [(0, 0), (1, 3), (8, 8)])
def test_recurrence_writes_its_outputs_alone(B, dtype, H, N, starts, ld, shift):  # noqa: F811
    S = 1 if starts is None else len(starts) - 1
    st = None if starts is None else torch.tensor(starts, dtype=torch.int32, device="cuda")
    G, V, D = (torch.randn(H, N, device="cuda").to(dtype) for _ in range(3))
    h0, dT = torch.randn(H, S, device="cuda"), torch.randn(H, S, device="cuda")
    cols = B.grim_glr_ckpt_cols(N)
    lo_, hi = (0, N) if starts is None else (starts[0], starts[-1])
    names = ("Y", "hT", "ckpt", "dG", "dV", "dh0")
    shapes = dict(Y=(N, dtype), hT=(S, F32), ckpt=(cols, F32), dG=(N, dtype), dV=(N, dtype), dh0=(S, F32))
    out = {n: framed(H, shapes[n][0], shapes[n][1], shapes[n][0] + (0 if n == "ckpt" else ld), shift) for n in names}
    plain = {n: torch.full((H, shapes[n][0]), MARK, device="cuda", dtype=shapes[n][1]) for n in names}
    for o in ({n: m for n, (m, _) in out.items()}, plain):
        B.grim_glr_seq(G, V, o["Y"], B.GRIM_GLR_GATE, st, h0, o["hT"], o["ckpt"])
        B.grim_glr_seq_grad(G, V, D, o["dG"], o["dV"], B.GRIM_GLR_GATE, o["ckpt"], st, h0, dT, o["dh0"])
    for n in names:
        assert out[n][1](), n
        if n != "ckpt":
            assert torch.equal(out[n][0], plain[n]), n
        if shapes[n][0] == N and n != "ckpt":
            assert (out[n][0][:, :lo_] == MARK).all() and (out[n][0][:, hi:] == MARK).all(), n


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M,N", [(1, 1), (9, 333), (3, 20000)])
def test_epilogue_grad_writes_its_outputs_alone(B, dtype, M, N):  # noqa: F811
    dY, P = torch.randn(M, N, device="cuda").to(dtype), torch.randn(M, N, device="cuda").to(dtype)
    whole = torch.full((M + 16,), MARK, device="cuda")
    dP, beside = framed(M, N, dtype, N + 5, 3)
    B.grim_epilogue_grad(dY, dP, B.GRIM_ACT_GELU, P, whole[8:8 + M])
    assert beside() and (whole[:8] == MARK).all() and (whole[8 + M:] == MARK).all() and (whole[8:8 + M] != MARK).all()


# ---------------------------------------------------------------------------------------- graphs and streams

@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n", [1, 9, 64, 264, 1000])
def test_linear_and_its_gradient_in_graphs_and_on_streams(B, n, bf16):  # noqa: F811
    """Captured and replayed on other values, and on a second stream: what the same calls give one after the other."""
    M, K, dt = 600, 512, BF16 if bf16 else F32
    W = gen.dense_weight(M, K, seed=41)
    mask = gen.bcr_mask(M, K, 8, 32, compression=4.0, dist="uniform", seed=42, stream=3)
    h = B.grim_bcr_pack(W, mask, 8, 32, int(bf16), 0)
    other = B.grim_bcr_pack(W, mask, 8, 32, int(bf16), 0)  # (a handle is used by one stream at a time)
    if bf16:
        B.grim_bcr_reserve(h, n)
        B.grim_bcr_reserve(other, n)
    X, R, D = (torch.randn(s, n, device="cuda").to(dt) for s in (K, M, M))
    b = torch.randn(M, device="cuda")

    def bufs():
        return [torch.zeros(M, n, device="cuda", dtype=dt) for _ in range(3)] + [torch.zeros(M, device="cuda")]

    def go(o, handle=h, stream=None):
        B.grim_bcr_linear(handle, X, o[0], b, B.GRIM_ACT_GELU, R, o[1], stream)
        B.grim_epilogue_grad(D, o[2], B.GRIM_ACT_GELU, o[1], o[3], stream)

    go(bufs())
    torch.cuda.synchronize()
    o, graph = bufs(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        go(o)
    side = torch.cuda.Stream()
    for _ in range(3):
        for t in (X, R, D, b):
            t.copy_(torch.randn_like(t))
        for t in o:
            t.zero_()
        graph.replay()
        want, there = bufs(), bufs()
        torch.cuda.synchronize()
        go(want)
        go(there, other, side)
        torch.cuda.synchronize()
        Wm = orc.masked_weight(W, mask, int(bf16))
        p = Wm @ num(X) + num(b)[:, None]
        scale = np.linalg.norm(Wm, axis=1)[:, None] * np.linalg.norm(num(X), axis=0)[None, :] + np.abs(num(b))[:, None]
        for got in (o, there, want):
            close(got[1], p, 1e-5 * scale, dt, "pre")
            close(got[0], lo.act("gelu", p) + num(R), 1.13 * 1e-5 * scale + 32 * U * (1 + np.abs(p)) + U * np.abs(num(R)), dt, "Y")
            q = num(got[1])  # (the gradient's own input)
            w = num(D) * lo.act_grad("gelu", q)
            bound = 48 * U * (1 + np.abs(q)) * np.abs(num(D))
            close(got[2], w, bound, dt, "dP")
            close(got[3], w.sum(1), bound.sum(1) + (n / 32 + 32) * U * np.abs(w).sum(1), F32, "dbias")
    assert B.grim_bcr_status(h) == B.GRIM_OK and B.grim_bcr_status(other) == B.GRIM_OK
    del graph
    B.grim_bcr_destroy(h)
    B.grim_bcr_destroy(other)


# ---------------------------------------------------------------------------------------- the gradient to X

def to_x_case(B, M, K, bh, bw, bf16, widths, rate=4):  # noqa: F811
    W = gen.dense_weight(M, K, seed=51)
    mask = gen.bcr_mask(M, K, bh, bw, compression=rate, dist="uniform", seed=52, stream=3)
    h = B.grim_bcr_pack(W, mask, bh, bw, int(bf16), B.GRIM_PACK_REORDER)
    t = B.grim_bcr_transpose(h, B.GRIM_PACK_REORDER)
    Wt = orc.masked_weight(W, mask, int(bf16)).T
    dt = BF16 if bf16 else F32
    for n in widths:
        if bf16 and n % 2:
            B.grim_bcr_reserve(t, n)
        dP = gen.normal_f32((M, n), 1.0, 53, n)
        dP = gen.bf16_representable(dP) if bf16 else dP
        R = torch.randn(K, n, device="cuda").to(dt)
        dX, beside = framed(K, n, dt, n + n % 3, n % 2)
        want = Wt @ dP.astype(np.float64)
        bound = 1e-5 * np.linalg.norm(Wt, axis=1)[:, None] * np.linalg.norm(dP.astype(np.float64), axis=0)[None, :]
        B.grim_bcr_spmm(t, dev(dP, dt), dX)
        close(dX, want, bound, dt, f"dX, {n} columns")
        B.grim_bcr_linear(t, dev(dP, dt), dX, residual=R)
        close(dX, want + num(R), bound + U * np.abs(num(R)), dt, f"dX + R, {n} columns")
        assert beside()
    assert B.grim_bcr_status(t) == B.GRIM_OK
    B.grim_bcr_destroy(t)
    B.grim_bcr_destroy(h)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("bh,bw", [(4, 16), (8, 32), (16, 64), (8, 17), (3, 24)])
@pytest.mark.parametrize("M,K", [(200, 336), (1024, 520), (333, 131)])
def test_gradient_to_x(B, M, K, bh, bw, bf16):  # noqa: F811
    to_x_case(B, M, K, bh, bw, bf16, (1, 3, 8, 16, 17, 40, 131, 264, 515))


@pytest.mark.parametrize("bf16", [False, True])
def test_gradient_to_x_with_many_block_columns(B, bf16):  # noqa: F811
    """2055 block columns of four: more than the slab kernel lists."""
    to_x_case(B, 8220, 70, 4, 16, bf16, (1, 5, 16, 33, 200))
